// Learned relative position bias by buckets, added to attention scores, and the gradient of its table.
//
//   y[b, h, q, k] = x[b, h, q, k] + table[bucket(q, k)][h]
//   grad_table[u][h] = sum over b and over the (q, k) of bucket u of grad_out[b, h, q, k]
//
// bucket(q, k) = buckets[d] with d = k - q + tq - 1, for sequences.  A map [tq, tk] (2-D windows) is the same thing with one query
// row of tq * tk keys, and that is how it comes in here.  A bucket outside 0 .. n_buckets - 1 adds nothing and has no gradient.
//
// Both kernels are bound by memory, so the buckets must cost nothing per element: they walk along the diagonals, on which
// d is constant.  Let o be the offset of a row (b, h, q) and V the elements of a 16-byte vector.  Element i of the vector
// V (floor((o + q) / V) + m) of the tensor has d = V m + i - c + tq - 1 where c = (o + q) mod V is the row's class.  So a
// thread that owns (m, c) meets the same V distances in every row of that class, over queries and samples: forward keeps
// their biases in registers, backward their sums, and both only load and add (and store) inside the loop.  The classes
// are taken one after the other; the rows of a class are every V-th row or sample, or whatever arithmetic gives.
//
// Work is cut into items: a head, a block of query rows, a chunk of vectors (`lanes` of them) and a part of the batch.
#include <math.h>

#include "s2a_launch.h"
#include "s2a_oct.cuh"

namespace s2a {
namespace {

constexpr uint32_t kThreads = 256, kMostThreads = 320;
constexpr uint32_t kTableBytes = 128 * 1024;  // shared memory for the tables of a backward CTA
constexpr int kAhead = 4;                     // rows whose loads a thread has in flight

struct BiasArgs {
  const void* x;           // x or grad_out
  void* y;                 // forward
  const void* table;       // forward
  const int32_t* buckets;  // [tq + tk - 1]
  float* partials;         // backward: [head][CTA of the head][n_buckets]
  uint64_t tk;             // up to 2^40 (a map)
  uint32_t batch, heads, tq;
  uint32_t n_buckets;
  uint32_t block;          // query rows of an item
  uint32_t blocks, chunks, parts;  // items of a head: blocks * chunks * parts
  uint32_t lanes;          // threads of a CTA along a chunk; the other factor of the threads runs along the batch
  uint32_t ctas_per_head;
  uint32_t tables;         // backward: warps that have a table
  uint32_t threads;        // of a CTA
  int by_batch;            // the inner loop runs over samples (few query rows), not over query rows
  // Along the inner loop the class moves by `step` = 2^shift * odd (mod V) from row to row: rows of one class come every `period` =
  // V / 2^shift rows, and there are some if the class differs from the first row's by a multiple of 2^shift.
  uint32_t period, shift, odd;
  int wdt;
};

// An item, and the thread's place in it.
struct Item {
  uint32_t h, q0, q1, b0, b1;
  int64_t m;       // the thread's vector, relative to the rows' floor((o + q) / V)
  int64_t d0;      // the distance index of shared slot 0 (see slot())
};
// Distance V m + i - c + tq - 1 lives in shared slot V lane + i - c + V - 1 >= 0, spread so that lanes V apart fall in
// different banks.
template <int V> __device__ __forceinline__ uint32_t slot(uint32_t k) { return k + k / V; }
template <int V> __device__ __forceinline__ uint32_t slot_of(uint32_t lane, int i, uint32_t c) {
  const uint32_t k = i + V - 1 - c;  // 0 .. 2 V - 2
  return lane * (V + 1) + k + (k >= V ? 1u : 0u);
}
template <int V> __host__ __device__ constexpr uint32_t slots(uint32_t lanes) { return lanes * V + V - 1; }
template <int V> __host__ __device__ constexpr uint32_t padded(uint32_t lanes) { return slots<V>(lanes) + slots<V>(lanes) / V + 1; }

template <int V>
__device__ __forceinline__ Item item_of(const BiasArgs& a, uint32_t h, uint64_t index, uint32_t lane) {
  Item t;
  t.h = h;
  const uint64_t place = a.parts == 1 ? index : index / a.parts;
  const uint32_t part = (uint32_t)(index - place * a.parts);
  const uint32_t block = a.blocks == 1 ? 0u : (uint32_t)(place / a.chunks), chunk = (uint32_t)(place - (uint64_t)block * a.chunks);
  t.q0 = block * a.block;
  t.q1 = min(a.tq, t.q0 + a.block);
  t.b0 = (uint32_t)((uint64_t)a.batch * part / a.parts);
  t.b1 = (uint32_t)((uint64_t)a.batch * (part + 1) / a.parts);
  // the lowest vector that a row of the block can need: k >= 0, i.e. V m >= c - q - (V - 1) with c >= 0, q <= q1 - 1
  const int64_t low = -(int64_t)((t.q1 - 1 + V - 1) / V) + (int64_t)chunk * a.lanes;
  t.m = low + lane;
  t.d0 = low * V - (V - 1) + (int64_t)a.tq - 1;
  return t;
}

// The first row of class c, counted from one of class c0; false if there is none.  r * 2^shift * odd = c - c0 (mod V) has the
// solution r = (c - c0) / 2^shift * odd (mod period): an odd number is its own inverse modulo 8.
template <int V>
__device__ __forceinline__ bool first_of_class(const BiasArgs& a, uint32_t c0, uint32_t c, uint32_t& r) {
  const uint32_t off = (c - c0) & (V - 1);
  r = ((off >> a.shift) * a.odd) & (a.period - 1);
  return (off & ((1u << a.shift) - 1u)) == 0;
}

// Calls body(n, e, e_step, k, k_step) for the runs of rows of class c that row-thread `row` of `rows` takes: n rows, the first
// with the thread's vector at element e of the tensor and key k (both may lie outside), the others e_step and k_step on.
template <int V, class Body>
__device__ __forceinline__ void walk(const BiasArgs& a, const Item& t, uint32_t c, uint32_t row, uint32_t rows, Body body) {
  const uint64_t slab = a.tq * a.tk, sample = slab * a.heads;
  uint32_t r;
  if (a.by_batch) {
    for (uint32_t q = t.q0; q < t.q1; ++q) {
      const uint64_t o = t.b0 * sample + t.h * slab + q * a.tk;
      if (!first_of_class<V>(a, (uint32_t)o + q, c, r)) continue;
      const uint32_t b = t.b0 + r + row * a.period, step = rows * a.period;  // samples b, b + step, ...
      if (b >= t.b1) continue;
      const int64_t k = t.m * V - c + q;
      body((int)((t.b1 - b + step - 1) / step), (int64_t)(o + (b - t.b0) * sample) + k, (int64_t)(step * sample), k, 0);
    }
  } else {
    for (uint32_t b = t.b0 + row; b < t.b1; b += rows) {
      const uint64_t o = b * sample + t.h * slab + t.q0 * a.tk;
      if (!first_of_class<V>(a, (uint32_t)o + t.q0, c, r) || t.q0 + r >= t.q1) continue;
      const int64_t k = t.m * V - c + t.q0 + r;  // query rows q0 + r, q0 + r + period, ...
      body((int)((t.q1 - t.q0 - r + a.period - 1) / a.period), (int64_t)(o + r * a.tk) + k, (int64_t)(a.period * (a.tk + 1)), k,
           (int)a.period);
    }
  }
}

// Keys k .. k + V - 1 against 0 .. tk - 1, in 32 bits: `at` counts from the run's first row (at most a block of rows on).
struct KeyRange {
  int low, high;  // a vector `at` keys on is wholly inside for low <= at <= high, wholly outside for at <= low - V, at >= high + V
  __device__ __forceinline__ KeyRange(int64_t k, uint64_t tk, int V) {
    const int64_t far = 1 << 30, hi = (int64_t)tk - V - k;
    low = (int)(-k > far ? far : (-k < -far ? -far : -k));
    high = (int)(hi > far ? far : (hi < -far ? -far : hi));
  }
  __device__ __forceinline__ bool inside(int at) const { return at >= low && at <= high; }
  __device__ __forceinline__ bool outside(int at, int V) const { return at <= low - V || at >= high + V; }
};

template <int DT>
__device__ __forceinline__ uint4 load_ends(const typename Io<DT>::T* x, int from, int to) {  // elements from .. to - 1 of a vector
  float f[kVec<DT>];
#pragma unroll
  for (int i = 0; i < kVec<DT>; ++i) f[i] = i >= from && i < to ? Io<DT>::widen(x[i]) : 0.0f;
  F2 v[kPairs<DT>];
#pragma unroll
  for (int i = 0; i < kPairs<DT>; ++i) v[i] = f2_pack(f[2 * i], f[2 * i + 1]);
  return narrow_piece<DT>(v);
}

// ---------------------------------------------------------------- forward
template <int DT>
__device__ __forceinline__ uint4 add_bias(const uint4& r, const float* bias) {
  F2 v[kPairs<DT>];
  widen_piece<DT>(r, v);
#pragma unroll
  for (int i = 0; i < kPairs<DT>; ++i) v[i] = f2_add(v[i], f2_pack(bias[2 * i], bias[2 * i + 1]));
  return narrow_piece<DT>(v);
}

template <int DT>
__global__ void __launch_bounds__(kMostThreads, 3) bias_fwd_kernel(BiasArgs a) {
  using T = typename Io<DT>::T;
  constexpr int V = kVec<DT>;
  extern __shared__ float bias_of[];  // by slot: the bias of each distance of the chunk
  enter_grid();
  const uint32_t lane = threadIdx.x % a.lanes, row = threadIdx.x / a.lanes, rows = blockDim.x / a.lanes;
  const uint32_t h = blockIdx.x / a.ctas_per_head, count = slots<V>(a.lanes);
  const uint64_t items = (uint64_t)a.blocks * a.chunks * a.parts;
  const int64_t distances = (int64_t)(a.tq + a.tk - 1);
  for (uint64_t index = blockIdx.x % a.ctas_per_head; index < items; index += a.ctas_per_head) {
    const Item t = item_of<V>(a, h, index, lane);
    __syncthreads();  // the previous item's biases have been read
    for (uint32_t k = threadIdx.x; k < count; k += blockDim.x) {
      const int64_t d = t.d0 + k;
      const int u = d >= 0 && d < distances ? a.buckets[d] : -1;
      bias_of[slot<V>(k)] = u >= 0 && (uint32_t)u < a.n_buckets ? load_param(a.table, (uint64_t)u * a.heads + h, a.wdt) : 0.0f;
    }
    __syncthreads();
#pragma unroll 1
    for (uint32_t c = 0; c < V; ++c) {
      walk<V>(a, t, c, row, rows, [&](int n, int64_t e, int64_t e_step, int64_t k, int k_step) {
        float bias[V];
#pragma unroll
        for (int i = 0; i < V; ++i) bias[i] = bias_of[slot_of<V>(lane, i, c)];
        const KeyRange range(k, a.tk, V);
        const T* x = (const T*)a.x + e;
        T* y = (T*)a.y + e;
        for (int j = 0, at = 0; j < n; j += kAhead, at += kAhead * k_step, x += kAhead * e_step, y += kAhead * e_step) {
          uint4 r[kAhead];
          if (j + kAhead <= n && at >= range.low && at + (kAhead - 1) * k_step <= range.high) {
#pragma unroll
            for (int s = 0; s < kAhead; ++s) r[s] = *(const uint4*)(x + s * e_step);
#pragma unroll
            for (int s = 0; s < kAhead; ++s) *(uint4*)(y + s * e_step) = add_bias<DT>(r[s], bias);
            continue;
          }
#pragma unroll
          for (int s = 0; s < kAhead; ++s)
            if (j + s < n && range.inside(at + s * k_step)) r[s] = *(const uint4*)(x + s * e_step);
#pragma unroll
          for (int s = 0; s < kAhead; ++s) {
            const int key = at + s * k_step;
            if (j + s >= n || range.outside(key, V)) continue;
            if (range.inside(key)) {
              *(uint4*)(y + s * e_step) = add_bias<DT>(r[s], bias);
            } else {  // an end of the row: element by element
              const int from = range.low - key, to = range.high + V - key;
#pragma unroll
              for (int i = 0; i < V; ++i)
                if (i >= from && i < to) y[s * e_step + i] = Io<DT>::narrow(Io<DT>::widen(x[s * e_step + i]) + bias[i]);
            }
          }
        }
      });
    }
  }
}

// ---------------------------------------------------------------- backward
// Adds one value per lane (bucket u, none for u < 0) to a warp's table.  Neighbouring lanes of one bucket are added up first
// (a segmented scan), then the last lane of each run adds its sum; runs of one bucket apart from each other take turns
// in lane order.  No atomics: the order is always the same.
__device__ __forceinline__ void table_add(float* table, int u, float v) {
  const unsigned all = 0xffffffffu;
  const uint32_t lane = threadIdx.x % 32;
  const int before = __shfl_up_sync(all, u, 1), after = __shfl_down_sync(all, u, 1);
  const bool head = lane == 0 || before != u, tail = lane == 31 || after != u;
  if (__any_sync(all, !head)) {
    const uint32_t heads = __ballot_sync(all, head);
    const uint32_t start = 31 - __clz(heads & (0xffffffffu >> (31 - lane)));  // where this lane's run begins
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const float w = __shfl_up_sync(all, v, o);
      if (lane >= start + o) v += w;
    }
  }
  const bool mine = tail && u >= 0;
  const unsigned peers = __match_any_sync(all, mine ? u : -1 - (int)lane);
  if (__all_sync(all, peers == (1u << lane))) {
    if (mine) table[u] += v;
    __syncwarp();
    return;
  }
  const int turn = __popc(peers & ((1u << lane) - 1u)), turns = __reduce_max_sync(all, turn);
  for (int k = 0; k <= turns; ++k) {
    if (mine && turn == k) table[u] += v;
    __syncwarp();
  }
}

template <int DT>
__global__ void __launch_bounds__(kMostThreads, 3) bias_bwd_kernel(BiasArgs a) {
  using T = typename Io<DT>::T;
  constexpr int V = kVec<DT>;
  extern __shared__ float shared[];  // [tables][n_buckets], then by row-thread and slot: the sum of each distance of the chunk
  enter_grid();
  const uint32_t lane = threadIdx.x % a.lanes, row = threadIdx.x / a.lanes, rows = blockDim.x / a.lanes, warp = threadIdx.x / 32;
  const uint32_t h = blockIdx.x / a.ctas_per_head, count = slots<V>(a.lanes), pad = padded<V>(a.lanes);
  const uint64_t items = (uint64_t)a.blocks * a.chunks * a.parts;
  const int64_t distances = (int64_t)(a.tq + a.tk - 1);
  float* sums = shared + a.tables * a.n_buckets;
  for (uint32_t i = threadIdx.x; i < a.tables * a.n_buckets; i += blockDim.x) shared[i] = 0.0f;
  for (uint64_t index = blockIdx.x % a.ctas_per_head; index < items; index += a.ctas_per_head) {
    const Item t = item_of<V>(a, h, index, lane);
    __syncthreads();  // the previous item's sums have been read
    for (uint32_t k = threadIdx.x; k < rows * pad; k += blockDim.x) sums[k] = 0.0f;
#pragma unroll 1
    for (uint32_t c = 0; c < V; ++c) {
      F2 acc[V / 2];
#pragma unroll
      for (int i = 0; i < V / 2; ++i) acc[i] = f2_both(0.0f);
      int any = 0;  // a class may have no rows
      walk<V>(a, t, c, row, rows, [&](int n, int64_t e, int64_t e_step, int64_t k, int k_step) {
        any = 1;
        const KeyRange range(k, a.tk, V);
        const T* x = (const T*)a.x + e;
        for (int j = 0, at = 0; j < n; j += kAhead, at += kAhead * k_step, x += kAhead * e_step) {
          uint4 r[kAhead];
          if (j + kAhead <= n && at >= range.low && at + (kAhead - 1) * k_step <= range.high) {
#pragma unroll
            for (int s = 0; s < kAhead; ++s) r[s] = *(const uint4*)(x + s * e_step);
          } else {
#pragma unroll
            for (int s = 0; s < kAhead; ++s) {
              const int key = at + s * k_step;
              r[s] = make_uint4(0, 0, 0, 0);
              if (j + s >= n || range.outside(key, V)) continue;
              if (range.inside(key)) r[s] = *(const uint4*)(x + s * e_step);
              else r[s] = load_ends<DT>(x + s * e_step, range.low - key, range.high + V - key);
            }
          }
#pragma unroll
          for (int s = 0; s < kAhead; ++s) {
            F2 v[V / 2];
            widen_piece<DT>(r[s], v);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) acc[i] = f2_add(acc[i], v[i]);
          }
        }
      });
      // the classes overlap: a slot belongs to neighbouring lanes in different classes
      if (!__syncthreads_or(any)) continue;
      float* mine = sums + row * pad;
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        float lo, hi;
        f2_unpack(acc[i], lo, hi);
        mine[slot_of<V>(lane, 2 * i, c)] += lo;
        mine[slot_of<V>(lane, 2 * i + 1, c)] += hi;
      }
    }
    __syncthreads();
    if (warp < a.tables) {
      float* table = shared + warp * a.n_buckets;
      for (uint32_t k0 = warp * 32; k0 < count; k0 += a.tables * 32) {
        const uint32_t k = k0 + threadIdx.x % 32;
        const int64_t d = t.d0 + k;
        int u = k < count && d >= 0 && d < distances ? a.buckets[d] : -1;
        if (u < 0 || (uint32_t)u >= a.n_buckets) u = -1;
        float v = 0.0f;
        if (u >= 0)
          for (uint32_t w = 0; w < rows; ++w) v += sums[w * pad + slot<V>(k)];
        table_add(table, u, v);
      }
    }
  }
  __syncthreads();
  float* part = a.partials + (uint64_t)blockIdx.x * a.n_buckets;
  for (uint32_t u = threadIdx.x; u < a.n_buckets; u += blockDim.x) {
    float s = 0.0f;
    for (uint32_t w = 0; w < a.tables; ++w) s += shared[w * a.n_buckets + u];
    part[u] = s;
  }
}

// [head][CTA of the head][n_buckets] -> grad_table[n_buckets][heads].  A CTA owns 32 buckets of one head; its eight
// warps take every eighth of the head's tables.
__global__ void __launch_bounds__(256) bias_table_kernel(const float* partials, uint32_t ctas_per_head, uint32_t n_buckets,
                                                         uint32_t heads, void* grad_table, int wdt) {
  __shared__ float sums[8][32];
  enter_grid();
  const uint32_t u = blockIdx.x * 32 + threadIdx.x % 32, w = threadIdx.x / 32, h = blockIdx.y;
  float t = 0.0f;
  if (u < n_buckets) {
#pragma unroll 4
    for (uint32_t j = w; j < ctas_per_head; j += 8) t += partials[((uint64_t)h * ctas_per_head + j) * n_buckets + u];
  }
  sums[w][threadIdx.x % 32] = t;
  __syncthreads();
  if (w == 0 && u < n_buckets) {
#pragma unroll
    for (int k = 1; k < 8; ++k) t += sums[k][threadIdx.x];
    store_param(grad_table, (uint64_t)u * heads + h, wdt, t);
  }
}

// ---------------------------------------------------------------- host side
uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// Cuts the work of every head into items, about `want` of them over all heads.
template <int V>
void cut(BiasArgs& a, uint64_t want) {
  const uint64_t per_head = ceil_div(want, a.heads);
  // query rows of an item: with many, the inner loop runs along the diagonals; with few, over the samples
  a.by_batch = a.tq < 4 * V;
  a.block = a.by_batch ? (a.tq < V ? a.tq : V) : 128;
  const uint32_t step = (uint32_t)((a.by_batch ? (uint64_t)a.heads * a.tq * a.tk : a.tk + 1) % V);
  a.shift = 0;
  while ((1u << a.shift) < V && (step >> a.shift) % 2 == 0) ++a.shift;
  a.period = V >> a.shift;
  a.odd = step >> a.shift;
  // the vectors that the rows of a block can need, whatever their class
  const auto vectors = [&] { return (a.tk + V - 2) / V + 1 + (a.block + V - 2) / V; };
  while (!a.by_batch && a.block > 32 && ceil_div(a.tq, a.block) * ceil_div(vectors(), kMostThreads) * a.batch < per_head) a.block /= 2;
  a.blocks = (uint32_t)ceil_div(a.tq, a.block);
  // the threads along them: a CTA's width with one row of threads, or a power of two with several side by side
  const uint64_t vecs = vectors();
  a.lanes = 8;
  while (a.lanes < 128 && a.lanes < vecs) a.lanes *= 2;
  if (vecs > 128) a.lanes = (uint32_t)ceil_div(ceil_div(vecs, ceil_div(vecs, kMostThreads)), 32) * 32;
  // fewer lanes (and more samples side by side) where the chunks are too few and the samples enough
  const uint64_t side = a.by_batch ? a.period * kAhead : 1;  // samples that keep one row of threads busy
  while (a.lanes > 32 && a.blocks * ceil_div(vecs, a.lanes) < per_head) {
    const uint32_t less = a.lanes > 128 ? 128 : a.lanes / 2;
    if (kThreads / less * side > a.batch) break;
    a.lanes = less;
  }
  a.threads = a.lanes > 128 ? a.lanes : kThreads;
  a.chunks = (uint32_t)ceil_div(vecs, a.lanes);
  const uint64_t most = ceil_div(a.batch, a.threads / a.lanes * side), parts = ceil_div(per_head, (uint64_t)a.blocks * a.chunks);
  a.parts = (uint32_t)(parts < 1 ? 1 : (parts < most ? parts : most));
  const uint64_t items = (uint64_t)a.blocks * a.chunks * a.parts, cap = 4 * per_head;
  a.ctas_per_head = (uint32_t)(items < cap ? items : cap);
}

BiasArgs shape_args(uint32_t batch, uint32_t heads, uint32_t tq, uint32_t tk, uint32_t n_buckets, bool by_distance) {
  BiasArgs a = {};
  a.batch = batch;
  a.heads = heads;
  a.tq = by_distance ? tq : 1;
  a.tk = by_distance ? tk : (uint64_t)tq * tk;
  a.n_buckets = n_buckets;
  return a;
}

constexpr uint64_t kFwdItems = 148 * 8;  // eight CTAs of 256 threads per SM of a B200
// The backward kernel writes a table per CTA: half as many CTAs, and fewer yet for tables of many buckets.
uint64_t bwd_items(uint32_t n_buckets) {
  const uint64_t most = (1ull << 23) / n_buckets;
  return most < 148 * 4 ? most : 148 * 4;
}

template <int DT>
cudaError_t launch_bias_fwd(BiasArgs& a, cudaStream_t st) {
  constexpr int V = kVec<DT>;
  cut<V>(a, kFwdItems);
  return launch_overlapped(bias_fwd_kernel<DT>, dim3(a.heads * a.ctas_per_head), a.threads, padded<V>(a.lanes) * sizeof(float), st, a);
}

template <int DT>
cudaError_t launch_bias_bwd(BiasArgs& a, cudaStream_t st) {
  constexpr int V = kVec<DT>;
  static std::atomic<uint64_t> ready = {};
  cut<V>(a, bwd_items(a.n_buckets));
  uint32_t tables = a.threads / 32;
  while (tables > 1 && (tables * a.n_buckets * sizeof(float) > kTableBytes || tables * 64 > slots<V>(a.lanes))) tables /= 2;
  a.tables = tables;
  const size_t smem = ((size_t)tables * a.n_buckets + (size_t)(a.threads / a.lanes) * padded<V>(a.lanes)) * sizeof(float);
  const cudaError_t e = allow_shared(bias_bwd_kernel<DT>, kTableBytes + 64 * 1024, ready);
  return e != cudaSuccess ? e : launch_overlapped(bias_bwd_kernel<DT>, dim3(a.heads * a.ctas_per_head), a.threads, smem, st, a);
}

}  // namespace

// The most CTAs over the element types and the two forms, which the size of the scratch does not tell apart.
uint32_t relbias_bwd_ctas(uint32_t batch, uint32_t heads, uint32_t tq, uint32_t tk, uint32_t n_buckets) {
  uint32_t most = 0;
  for (int form = 0; form < 2; ++form) {
    BiasArgs a = shape_args(batch, heads, tq, tk, n_buckets, form != 0);
    cut<kVec<kF32>>(a, bwd_items(n_buckets));
    most = a.ctas_per_head > most ? a.ctas_per_head : most;
    cut<kVec<kBF16>>(a, bwd_items(n_buckets));
    most = a.ctas_per_head > most ? a.ctas_per_head : most;
  }
  return heads * most;
}

cudaError_t launch_relbias_fwd(int dt, int wdt, const void* x, const void* table, const int32_t* buckets, int by_distance,
                               void* y, uint32_t batch, uint32_t heads, uint32_t tq, uint32_t tk, uint32_t n_buckets,
                               cudaStream_t st) {
  BiasArgs a = shape_args(batch, heads, tq, tk, n_buckets, by_distance != 0);
  a.x = x;
  a.y = y;
  a.table = table;
  a.buckets = buckets;
  a.wdt = wdt;
  return dt == kF32 ? launch_bias_fwd<kF32>(a, st) : launch_bias_fwd<kBF16>(a, st);
}

cudaError_t launch_relbias_bwd(int dt, int wdt, const void* g, const int32_t* buckets, int by_distance, void* grad_table,
                               float* scratch, uint32_t batch, uint32_t heads, uint32_t tq, uint32_t tk, uint32_t n_buckets,
                               cudaStream_t st) {
  if ((uint64_t)batch * tq * tk == 0)  // a sum over nothing
    return cudaMemsetAsync(grad_table, 0, (size_t)n_buckets * heads * (wdt == kF32 ? 4u : 2u), st);
  BiasArgs a = shape_args(batch, heads, tq, tk, n_buckets, by_distance != 0);
  a.x = g;
  a.buckets = buckets;
  a.partials = scratch;
  const cudaError_t e = dt == kF32 ? launch_bias_bwd<kF32>(a, st) : launch_bias_bwd<kBF16>(a, st);
  if (e != cudaSuccess) return e;
  return launch_overlapped(bias_table_kernel, dim3((n_buckets + 31) / 32, heads), 256, 0, st, scratch, a.ctas_per_head,
                           n_buckets, heads, grad_table, wdt);
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
