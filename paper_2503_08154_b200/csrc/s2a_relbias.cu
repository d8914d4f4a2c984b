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
// their biases in registers, backward their sums, and inside the loop both only load and add (and store).  The classes are
// taken one after the other.
//
// Work is cut into items: a head, a block of query rows, a chunk of vectors (`lanes` of them) and a part of the batch.
//
// What it measures on a B200 (6.57 TB/s copy rate), bfloat16: [64, 12, 197, 197] under a map of 732 buckets, forward 25.0 us (4.8 TB/s:
// 18 us of walking, which is the copy rate, after the look-up of the chunk's biases, and the launch), one sample of [16, 1025, 1025] 25 us
// (2.9 TB/s: bias_fwd_few_kernel, element by element: 24 instructions a warp and 32 elements, 58 % of the issue slots, and the wait for
// the bucket before the bias), backward 19.3 us (3.1 TB/s: about 13 of walking, the rest setup, tables and the second kernel), one
// sample of [16, 1025, 1025] 100 us (bias_bwd_few_kernel says why); by distance [64, 12, 197, 197] forward 38 us (4.1 TB/s), backward 28 us, [16, 16,
// 577, 577] 81 us (4.2 TB/s) and 41 us, [2, 16, 2048, 2048] 106 us (5.1 TB/s) and 53 us (5.1 TB/s): a row of an odd width is cut in two
// vectors, and its classes are all eight.  Looking the bucket of every element up where it is added costs 200 us
// there.  Measured and not kept: the rows through a ring of cp.async as in layer norm (92 us: the bookkeeping of a row's place
// outweighs the add), eight rows ahead in forward (spills, 33 us), rows asked for in L2 before the forward kernel's look-up (no gain).
#include <math.h>

#include <numeric>

#include "s2a_launch.h"
#include "s2a_oct.cuh"

namespace s2a {
namespace {

constexpr int kAheadFwd = 4, kAheadBwd = 6;  // rows of a run whose loads a thread has in flight
constexpr uint32_t kThreads = 256, kMostThreads = 320;
constexpr uint32_t kThreadsPerSm = 1024;     // at 64 registers a thread
constexpr int kAnnounced = 8;                // rows of an item's first run that are asked for before its shared memory is set up
constexpr int kStaged = 5;                   // slots that a thread looks up at a time
// bias_fwd_few_kernel and bias_bwd_few_kernel.  Up to so many samples they are faster than the diagonals, beyond that not always.
// Forward, [B, 12, 401, 401] bfloat16: B = 2: 8.4 us against 14.4, 4: 12.3 against 15.6, 8: 20.2 against 18.7; [1, 16, 1025, 1025] 25 against
// 75.  Backward, the same: 2: 18 against 34, 4: 21 against 35, 8: 26 against 37; [64, 12, 197, 197] 27.5 against 19.3; [1, 16, 1025, 1025] 100
// against 243.  Backward with larger tables, of which fewer warps have one (16 at 2,601 buckets, 8 at 5,329, 4 at 9,025 to 11,264), windows of
// 12 heads, bfloat16, one and eight samples: 2,601 buckets 29 us against 82 and 61 against 93; 5,329: 175 against 438 and 407 against
// 502; 6,561: 343 against 574 and 799 against 645; 7,225: 412 against 1314 and 967 against 1440; 9,025: 934 against 1361 and 2142 against 1456; 10,609:
// 1282 against 3899 and 2940 against 4084.  With 3 heads they are ahead everywhere (9,025 buckets: 246 against 529, 540 against 559), in binary32 up to
// six samples.  So from 6,000 buckets on the border lies anywhere between two samples and beyond eight, with how the
// diagonals' tables happen to fit an SM; eight loses up to 1.5 times there and wins up to 2.5 times.
constexpr uint32_t kFewSamplesFwd = 4, kFewSamplesBwd = 8;
constexpr uint32_t kFewThreads = 512, kFewPerSm = 2;  // four keys and three or four CTAs an SM: 28 to 30 us
constexpr int kFewKeys = 8;                           // keys of a thread in flight
constexpr uint32_t kColumnBuckets = 12288;            // of a column in 48 KB
constexpr uint32_t kFewTableBytes = 220 * 1024;       // shared memory of an SM for the tables of bias_bwd_few_kernel
constexpr uint32_t kTableBytes = 64 * 1024;  // shared memory for the tables of a backward CTA, beyond the first table

struct BiasArgs {
  const void* x;           // x or grad_out
  void* y;                 // forward
  const void* table;       // forward
  const int32_t* buckets;  // [tq + tk - 1]
  float* partials;         // backward: [head][CTA of the head][n_buckets]
  uint64_t tk;             // up to 2^36 (a map)
  uint64_t slab, sample;   // elements of one (b, h), of one b
  uint32_t batch, heads, tq;
  uint32_t n_buckets;
  uint32_t block;          // query rows of an item
  uint32_t part;           // samples of an item
  uint32_t chunks, parts, items;  // chunks of vectors, parts of the batch; items of a head: (query blocks) * chunks * parts
  uint32_t lanes, rows;    // threads of a CTA along a chunk, and along the batch
  uint32_t ctas_per_head, threads;
  uint32_t tables;         // backward: warps that have a table
  int column;              // bias_fwd_few_kernel: the head's column of the table comes into shared memory first
  int by_batch;            // the inner loop runs over samples (few query rows), not over query rows
  int wdt;
  // Along the inner loop the class moves by `step` = 2^shift * odd (mod V) from row to row: rows of one class come every `period` =
  // V / 2^shift rows, and there are some if the class differs from the first row's by a multiple of 2^shift.
  uint32_t step, period, period_log, shift, odd;
  uint32_t classes;        // with one query row the classes are those of the samples; with more, any may occur
  int64_t row_step;        // elements between the rows of a run, and the keys that the thread's vector moves by
  int key_step;
};

// An item, and the thread's place in it.
struct Item {
  uint32_t queries, samples;  // of the item
  uint32_t c0;                // class of its first row
  // The thread's vector in the first row, were that row of class 0: its element in the tensor, and the keys it is from being
  // wholly inside the row, V m + q0 >= 0 and <= tk - V.
  int64_t e;
  int key_low, key_high;
  // Shared slot k (see slot()) is distance d0 + k: its bucket is lut[k], for low <= k < high.
  const int32_t* lut;
  int low, high;
};
// Distance V m + i - c + tq - 1 lives in slot V lane + i - c + V - 1 >= 0 of the chunk.
template <int V> __host__ __device__ constexpr uint32_t slots(uint32_t lanes) { return lanes * V + V - 1; }
// In the forward kernel's shared memory the slots are spread so that lanes V apart fall in different banks.
template <int V> __device__ __forceinline__ uint32_t spread(uint32_t k) { return k + k / V; }
template <int V> __host__ __device__ constexpr uint32_t spread_slots(uint32_t lanes) { return slots<V>(lanes) + slots<V>(lanes) / V + 1; }

__device__ __forceinline__ int clamp_int(int64_t v) {
  const int64_t far = 1 << 30;
  return (int)(v > far ? far : (v < -far ? -far : v));
}

template <int V>
__device__ __forceinline__ Item item_of(const BiasArgs& a, uint32_t h, uint32_t index, uint32_t lane) {
  Item t;
  const uint32_t place = a.parts == 1 ? index : index / a.parts, part = index - place * a.parts;
  const uint32_t block = place / a.chunks, chunk = place - block * a.chunks;
  const uint32_t q0 = block * a.block, b0 = part * a.part;
  t.queries = min(a.tq - q0, a.block);
  t.samples = b0 < a.batch ? min(a.batch - b0, a.part) : 0;
  const uint64_t first = b0 * a.sample + h * a.slab + q0 * a.tk;
  t.c0 = ((uint32_t)first + q0) & (V - 1);
  // the lowest vector that a row of the block can need: k >= 0, i.e. V m >= c - q - (V - 1) with c >= 0, q < q0 + queries
  const int64_t lowest = (int64_t)chunk * a.lanes - (int64_t)((q0 + t.queries + V - 2) / V);
  const int64_t k = (lowest + lane) * V + q0;
  t.e = (int64_t)first + k;
  t.key_low = clamp_int(-k);
  t.key_high = clamp_int((int64_t)a.tk - V - k);
  const int64_t d0 = lowest * V - (V - 1) + (int64_t)a.tq - 1;
  t.lut = a.buckets + d0;
  t.low = clamp_int(-d0);
  t.high = clamp_int((int64_t)(a.tq + a.tk) - 1 - d0);
  return t;
}

// The bucket of slot k, -1 for none (and for k < 0).
__device__ __forceinline__ int bucket_of(const BiasArgs& a, const Item& t, int k) {
  const int u = k >= 0 && k >= t.low && k < t.high ? t.lut[k] : -1;
  return (uint32_t)u < a.n_buckets ? u : -1;
}

// The runs of an item as one thread takes them, class by class.  A run: the rows of one class along the inner loop (samples or
// query rows), row_step elements apart, of which the thread's vector moves by key_step keys.
template <int V>
struct Runs {
  uint32_t i, c;    // the class, by number and as it is
  uint32_t o;       // a query row of the item (by_batch) or a sample
  int n;            // rows of the run
  int low, high;    // row j's vector is wholly inside its row for low <= j * key_step <= high, wholly outside for j * key_step <= low - V
                    // and for j * key_step >= high + V
  int64_t e;        // the first row's element

  __device__ __forceinline__ void start(const BiasArgs& a, const Item& t, uint32_t row) {
    i = row < a.rows ? 0 : a.classes;  // threads may be left over
    o = a.by_batch ? 0 : row;
    seek(a, t, row);
  }
  __device__ __forceinline__ bool done(const BiasArgs& a) const { return i >= a.classes; }
  __device__ __forceinline__ void next(const BiasArgs& a, const Item& t, uint32_t row) {
    o += a.by_batch ? 1 : a.rows;
    seek(a, t, row);
  }

  // The first run at or after run o of class i.
  __device__ __forceinline__ void seek(const BiasArgs& a, const Item& t, uint32_t row) {
    for (; i < a.classes; ++i, o = a.by_batch ? 0 : row) {
      c = a.tq == 1 ? (t.c0 + i * a.step) & (V - 1) : i;
      const uint32_t end = a.by_batch ? t.queries : t.samples, hop = a.by_batch ? 1 : a.rows;
      for (; o < end; o += hop) {
        // The run's first row: r * 2^shift * odd = c - (class of row 0) (mod V) has the solution
        // r = (c - class) / 2^shift * odd (mod period), as an odd number is its own inverse modulo 8.
        const uint32_t off = (c - t.c0 - o * (a.by_batch ? (uint32_t)a.tk + 1 : (uint32_t)a.sample)) & (V - 1);
        if (off & ((1u << a.shift) - 1u)) continue;
        uint32_t r = ((off >> a.shift) * a.odd) & (a.period - 1);
        uint32_t q = r;
        if (a.by_batch) {  // samples r + row * period, + rows * period, ...
          r += row * a.period;
          q = o;
          n = r < t.samples ? (int)((t.samples - r - 1) / (a.rows * a.period)) + 1 : 0;
        } else {           // query rows r, + period, ...
          n = r < t.queries ? (int)((t.queries - r - 1) >> a.period_log) + 1 : 0;
        }
        if (n == 0) continue;
        e = t.e + (int64_t)((a.by_batch ? r : o) * a.sample + q * (a.tk + 1)) - c;
        low = t.key_low - (int)(q - c);
        high = t.key_high - (int)(q - c);
        return;
      }
    }
  }

  // Asks for the run's first rows in L2, ahead of the loop that loads them.
  template <typename T>
  __device__ __forceinline__ void announce(const BiasArgs& a, const T* x) const {
    if (done(a)) return;
#pragma unroll 1
    for (int j = 0; j < kAnnounced && j < n; ++j)
      if (j * a.key_step >= low && j * a.key_step <= high) asm volatile("prefetch.global.L2 [%0];" ::"l"(x + e + j * a.row_step));
  }

  // The rows of the run that the vector meets.  Along the samples (key_step 0) all of them, in one way: j = 0 .. in1 - 1, all
  // whole or all cut.  Along the query rows whole ones, in0 <= j < in1, and cut ones, the other j of any0 <= j < any1.
  __device__ __forceinline__ void meets(const BiasArgs& a, int& any0, int& any1, int& in0, int& in1, bool& cut) const {
    if (a.by_batch) {
      any0 = any1 = in0 = 0;
      in1 = low < V && high > -V ? n : 0;
      cut = low > 0 || high < 0;
    } else {
      const int log = (int)a.period_log, up = a.key_step - 1;
      any0 = max(0, (low - V + 1 + up) >> log);
      any1 = max(any0, min(n, ((high + V - 1) >> log) + 1));
      in0 = max(any0, (low + up) >> log);
      in1 = min(any1, (high >> log) + 1);
      if (in0 >= in1) in0 = in1 = any1;
      cut = false;
    }
  }
};

// Loads elements from .. to - 1 of a vector, zeros in place of the others; one by one, as the rest of the vector is another row's, or
// lies after the tensor.
template <int DT>
__device__ __forceinline__ uint4 load_ends(const typename Io<DT>::T* x, int from, int to) {
  uint32_t w[kVec<DT>];
#pragma unroll
  for (int i = 0; i < kVec<DT>; ++i) {
    w[i] = 0;
    if (i < from || i >= to) continue;
    if constexpr (DT == kF32) w[i] = __float_as_uint(x[i]);
    else w[i] = __bfloat16_as_ushort(x[i]);
  }
  if constexpr (DT == kF32) return make_uint4(w[0], w[1], w[2], w[3]);
  else return make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
}

// The vector at x, of which elements from .. to - 1 count: whole where the tensor holds it whole (the rest is another row's), the
// tensor's last one element by element.
template <int DT>
__device__ __forceinline__ uint4 load_cut(const typename Io<DT>::T* x, const typename Io<DT>::T* end, int from, int to) {
  return x + kVec<DT> <= end ? *(const uint4*)x : load_ends<DT>(x, from, to);
}
// Elements from .. to - 1 of a vector, zeros in place of the others.
template <int DT>
__device__ __forceinline__ uint4 keep_elements(const uint4& v, int from, int to) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < kVec<DT>; ++i)
    if (i < from || i >= to) w[DT == kF32 ? i : i / 2] &= DT == kF32 ? 0u : (i % 2 ? 0x0000ffffu : 0xffff0000u);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Stores elements from .. to - 1 of a vector.
template <int DT>
__device__ __forceinline__ void store_ends(typename Io<DT>::T* y, const uint4& v, int from, int to) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < kVec<DT>; ++i) {
    if (i < from || i >= to) continue;
    if constexpr (DT == kF32) y[i] = __uint_as_float(w[i]);
    else y[i] = __ushort_as_bfloat16((unsigned short)(w[i / 2] >> (16 * (i % 2))));
  }
}

// ---------------------------------------------------------------- forward
template <int DT>
__device__ __forceinline__ uint4 add_bias(const uint4& r, const F2* bias) {
  F2 v[kPairs<DT>];
  widen_piece<DT>(r, v);
#pragma unroll
  for (int i = 0; i < kPairs<DT>; ++i) v[i] = f2_add(v[i], bias[i]);
  return narrow_piece<DT>(v);
}

template <int DT>
__global__ void __launch_bounds__(kMostThreads, 3) bias_fwd_kernel(BiasArgs a) {
  using T = typename Io<DT>::T;
  constexpr int V = kVec<DT>;
  extern __shared__ float bias_of[];  // by slot
  enter_grid();
  const int64_t to_y = (const T*)a.y - (const T*)a.x;  // both on the 16-byte grid
  const uint32_t row = threadIdx.x / a.lanes, lane = threadIdx.x - row * a.lanes, h = blockIdx.y, count = slots<V>(a.lanes);
  for (uint32_t index = blockIdx.x; index < a.items; index += gridDim.x) {
    const Item t = item_of<V>(a, h, index, lane);
    if (index != blockIdx.x) __syncthreads();  // the previous item's biases have been read
    // several at a time: the two dependent loads of a slot are waited for once
    for (uint32_t k = threadIdx.x; k < count; k += kStaged * a.threads) {
      int u[kStaged];
      float v[kStaged];
#pragma unroll
      for (int i = 0; i < kStaged; ++i) u[i] = bucket_of(a, t, k + i * a.threads < count ? (int)(k + i * a.threads) : -1);
#pragma unroll
      for (int i = 0; i < kStaged; ++i) v[i] = u[i] >= 0 ? load_param(a.table, (uint64_t)u[i] * a.heads + h, a.wdt) : 0.0f;
#pragma unroll
      for (int i = 0; i < kStaged; ++i)
        if (k + i * a.threads < count) bias_of[spread<V>(k + i * a.threads)] = v[i];
    }
    __syncthreads();
    Runs<V> run;
#pragma unroll 1
    for (run.start(a, t, row); !run.done(a); run.next(a, t, row)) {
      int any0, any1, in0, in1;
      bool cut;
      run.meets(a, any0, any1, in0, in1, cut);
      if (any0 >= any1 && in0 >= in1) continue;
      F2 bias[V / 2];
      const uint32_t k = lane * V + V - 1 - run.c;
#pragma unroll
      for (int i = 0; i < V / 2; ++i) bias[i] = f2_pack(bias_of[spread<V>(k + 2 * i)], bias_of[spread<V>(k + 2 * i + 1)]);
      const T *x = (const T*)a.x + run.e + in0 * a.row_step, *end = (const T*)a.x + a.batch * a.sample;
      // A cut vector is read whole, as its other elements are a neighbouring row's; only the tensor's last may not lie in it.
      int left = in1 - in0;
      const bool beyond = cut && x + (left - 1) * a.row_step + V > end;
      if (beyond) --left;
#pragma unroll 1
      for (; left > 0; left -= kAheadFwd, x += kAheadFwd * a.row_step) {
        uint4 r[kAheadFwd];
#pragma unroll
        for (int s = 0; s < kAheadFwd; ++s)
          if (s < left) r[s] = *(const uint4*)(x + s * a.row_step);
#pragma unroll
        for (int s = 0; s < kAheadFwd; ++s) {
          if (s >= left) break;
          const uint4 w = add_bias<DT>(r[s], bias);
          T* y = (T*)(x + s * a.row_step + to_y);
          if (cut) store_ends<DT>(y, w, run.low, run.high + V);
          else *(uint4*)y = w;
        }
      }
      if (beyond) {
        const T* last = (const T*)a.x + run.e + (in1 - 1) * a.row_step;
        store_ends<DT>((T*)(last + to_y), add_bias<DT>(load_ends<DT>(last, run.low, run.high + V), bias), run.low, run.high + V);
      }
      // the cut rows: a few before the whole ones and a few after
      const int before = in0 - any0, cuts = before + any1 - in1;
#pragma unroll 1
      for (int j0 = 0; j0 < cuts; j0 += 2) {
        uint4 r[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int j = j0 + s < before ? any0 + j0 + s : in1 + j0 + s - before, moved = j * a.key_step;
          if (j < any1) r[s] = load_cut<DT>((const T*)a.x + run.e + j * a.row_step, end, run.low - moved, run.high + V - moved);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int j = j0 + s < before ? any0 + j0 + s : in1 + j0 + s - before, moved = j * a.key_step;
          if (j < any1) store_ends<DT>((T*)a.y + run.e + j * a.row_step, add_bias<DT>(r[s], bias), run.low - moved, run.high + V - moved);
        }
      }
    }
  }
}

// Maps with few samples: there is little for a bias to be kept for, and the way of a chunk through shared memory and the classes
// costs more than the elements.  Here neighbouring threads take neighbouring keys, one by one, whatever their alignment, and look
// a key's bias up once for all samples.  The buckets of neighbouring keys are mostly neighbours too, but their places in the table
// are `heads` apart, a line for every lane or two: so a CTA that looks up more keys than the table has buckets copies its
// head's column into shared memory first.
template <int DT>
__global__ void __launch_bounds__(kFewThreads, kFewPerSm) bias_fwd_few_kernel(BiasArgs a) {
  using T = typename Io<DT>::T;
  extern __shared__ float column[];  // by bucket
  enter_grid();
  const uint32_t h = blockIdx.y;
  if (a.column) {
#pragma unroll 4
    for (uint32_t u = threadIdx.x; u < a.n_buckets; u += kFewThreads) column[u] = load_param(a.table, (uint64_t)u * a.heads + h, a.wdt);
    __syncthreads();
  }
  for (uint64_t k0 = (uint64_t)blockIdx.x * kFewKeys * kFewThreads; k0 < a.tk; k0 += (uint64_t)gridDim.x * kFewKeys * kFewThreads) {
    const uint64_t k = k0 + threadIdx.x, first = h * a.slab + k;
    const int left = clamp_int((int64_t)(a.tk - k0) - threadIdx.x);  // key k + i * kFewThreads is there if i * kFewThreads < left
    const T* x = (const T*)a.x + first;
    T* y = (T*)a.y + first;
    int u[kFewKeys];
    T v[kFewKeys];
    float bias[kFewKeys];
#pragma unroll
    for (int i = 0; i < kFewKeys; ++i) u[i] = i * (int)kFewThreads < left ? a.buckets[k + i * kFewThreads] : -1;
#pragma unroll
    for (int i = 0; i < kFewKeys; ++i)
      if (i * (int)kFewThreads < left) v[i] = x[i * kFewThreads];
#pragma unroll
    for (int i = 0; i < kFewKeys; ++i)
      bias[i] = (uint32_t)u[i] >= a.n_buckets ? 0.0f : (a.column ? column[u[i]] : load_param(a.table, (uint64_t)u[i] * a.heads + h, a.wdt));
    for (uint32_t b = 0;;) {
#pragma unroll
      for (int i = 0; i < kFewKeys; ++i)
        if (i * (int)kFewThreads < left) y[i * kFewThreads] = Io<DT>::narrow(Io<DT>::widen(v[i]) + bias[i]);
      if (++b == a.batch) break;
      x += a.sample;
      y += a.sample;
#pragma unroll
      for (int i = 0; i < kFewKeys; ++i)
        if (i * (int)kFewThreads < left) v[i] = x[i * kFewThreads];
    }
  }
}

// ---------------------------------------------------------------- backward
// Adds one value per lane (bucket u, none for u < 0) to a warp's table.  Neighbouring lanes of one bucket are added up first
// (a segmented scan), and the last lane of each run adds its sum; runs of one bucket apart from each other take turns in
// lane order.  No atomics: the order is always the same.  Whether two runs meet is found by writing: each lane leaves its number at
// its bucket's tag and looks whether it is still there (__match_any_sync on 32 different buckets takes about 480 cycles, this about
// 50).  Which of two lanes a tag keeps does not matter.
__device__ __forceinline__ void table_add(float* table, uint8_t* tags, int u, float v) {
  const unsigned all = 0xffffffffu;
  const uint32_t lane = threadIdx.x % 32;
  const int before = __shfl_up_sync(all, u, 1), after = __shfl_down_sync(all, u, 1);
  const bool head = lane == 0 || before != u, tail = lane == 31 || after != u;
  const uint32_t heads = __ballot_sync(all, head);
  if (heads != all) {
    const uint32_t start = 31 - __clz(heads & (0xffffffffu >> (31 - lane)));  // where this lane's run begins
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const float w = __shfl_up_sync(all, v, o);
      if (lane >= start + o) v += w;
    }
  }
  const bool mine = tail && u >= 0;
  if (mine) tags[u] = (uint8_t)lane;
  __syncwarp();
  const bool met = mine && tags[u] != lane;
  if (!__any_sync(all, met)) {
    if (mine) table[u] += v;
    __syncwarp();
    return;
  }
  const unsigned peers = __match_any_sync(all, mine ? u : -1 - (int)lane);
  const int turn = __popc(peers & ((1u << lane) - 1u)), turns = __reduce_max_sync(all, turn);
  for (int k = 0; k <= turns; ++k) {
    if (mine && turn == k) table[u] += v;
    __syncwarp();
  }
}

// The sum of a CTA's tables, for bias_table_kernel.
__device__ __forceinline__ void write_partials(const BiasArgs& a, const float* tables) {
  float* part = a.partials + ((uint64_t)blockIdx.y * gridDim.x + blockIdx.x) * a.n_buckets;
  for (uint32_t u = threadIdx.x; u < a.n_buckets; u += a.threads) {
    float s = 0.0f;
    for (uint32_t w = 0; w < a.tables; ++w) s += tables[w * a.n_buckets + u];
    part[u] = s;
  }
}

template <int DT>
__device__ __forceinline__ void add_vector(F2* acc, const uint4& r) {
  F2 v[kPairs<DT>];
  widen_piece<DT>(r, v);
#pragma unroll
  for (int i = 0; i < kPairs<DT>; ++i) acc[i] = f2_add(acc[i], v[i]);
}

template <int DT>
__global__ void __launch_bounds__(kMostThreads, 3) bias_bwd_kernel(BiasArgs a) {
  using T = typename Io<DT>::T;
  constexpr int V = kVec<DT>;
  // [2 V - 1][stride]: a thread's sums of the distances V lane + 0 .. 2 V - 2 that its vector has in one class or another.
  // [tables][n_buckets]; [slots] the buckets; [tables][n_buckets] the tables' tags.
  extern __shared__ __align__(16) float sums[];
  enter_grid();
  const uint32_t row = threadIdx.x / a.lanes, lane = threadIdx.x - row * a.lanes, warp = threadIdx.x / 32, h = blockIdx.y;
  const uint32_t count = slots<V>(a.lanes);
  const uint32_t stride = a.threads + 32 / V;  // so that the sums of 32 neighbouring distances lie in 32 banks
  float* tables = sums + (2 * V - 1) * stride;
  int32_t* ids = (int32_t*)(tables + a.tables * a.n_buckets);
  uint8_t* tags = (uint8_t*)(ids + count);
  for (uint32_t index = blockIdx.x; index < a.items; index += gridDim.x) {
    const Item t = item_of<V>(a, h, index, lane);
    Runs<V> run;
    run.start(a, t, row);
    run.announce(a, (const T*)a.x);
    const bool first = index == blockIdx.x;
    if (!first) __syncthreads();  // the previous item's sums have been read
    const uint32_t zeros = (2 * V - 1) * stride + (first ? a.tables * a.n_buckets : 0);  // the tables once, the sums each time
    for (uint32_t i = threadIdx.x; i < zeros / 4; i += a.threads) ((float4*)sums)[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (threadIdx.x < zeros % 4) sums[zeros / 4 * 4 + threadIdx.x] = 0.0f;
    // the buckets come while the rows do
    for (uint32_t k = threadIdx.x; k < count; k += a.threads) {
      if ((int)k >= t.low && (int)k < t.high) copy_async<4>(ids + k, t.lut + k);
      else ids[k] = -1;
    }
    copy_commit();
    __syncthreads();
#pragma unroll 1
    for (; !run.done(a); run.next(a, t, row)) {
      int any0, any1, in0, in1;
      bool cut;
      run.meets(a, any0, any1, in0, in1, cut);
      if (any0 >= any1 && in0 >= in1) continue;
      F2 acc[V / 2];
#pragma unroll
      for (int i = 0; i < V / 2; ++i) acc[i] = f2_both(0.0f);
      const T *x = (const T*)a.x + run.e + in0 * a.row_step, *end = (const T*)a.x + a.batch * a.sample;
      // A cut vector is added whole, and the sums of the elements outside the row dropped at the end; only the tensor's last
      // vector may not lie in it.
      int left = in1 - in0;
      const bool beyond = cut && x + (left - 1) * a.row_step + V > end;
      if (beyond) --left;
#pragma unroll 1
      for (; left >= kAheadBwd; left -= kAheadBwd, x += kAheadBwd * a.row_step) {
        uint4 r[kAheadBwd];
#pragma unroll
        for (int s = 0; s < kAheadBwd; ++s) r[s] = *(const uint4*)(x + s * a.row_step);
#pragma unroll
        for (int s = 0; s < kAheadBwd; ++s) add_vector<DT>(acc, r[s]);
      }
      if (left > 0) {
        uint4 r[kAheadBwd - 1];
#pragma unroll
        for (int s = 0; s < kAheadBwd - 1; ++s) r[s] = s < left ? *(const uint4*)(x + s * a.row_step) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int s = 0; s < kAheadBwd - 1; ++s) add_vector<DT>(acc, r[s]);
      }
      if (beyond) add_vector<DT>(acc, load_ends<DT>((const T*)a.x + run.e + (in1 - 1) * a.row_step, run.low, run.high + V));
      // the cut rows: a few before the whole ones and a few after
      const int before = in0 - any0, cuts = before + any1 - in1;
#pragma unroll 1
      for (int j0 = 0; j0 < cuts; j0 += 2) {
        uint4 r[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const int j = j0 + s < before ? any0 + j0 + s : in1 + j0 + s - before, moved = j * a.key_step;
          r[s] = make_uint4(0, 0, 0, 0);
          if (j < any1)
            r[s] = keep_elements<DT>(load_cut<DT>((const T*)a.x + run.e + j * a.row_step, end, run.low - moved, run.high + V - moved),
                                     run.low - moved, run.high + V - moved);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) add_vector<DT>(acc, r[s]);
      }
      float* mine = sums + (V - 1 - run.c) * stride + threadIdx.x;  // the distances V lane + i - c + V - 1
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float lo, hi;
        f2_unpack(acc[i / 2], lo, hi);
        const float v = i % 2 ? hi : lo;
        mine[i * stride] += !cut || (i >= run.low && i < run.high + V) ? v : 0.0f;
      }
    }
    copy_wait<0>();
    __syncthreads();
    if (warp < a.tables) {
      // the distance of slot k is number k - V l of thread l for l = k / V, and of the one before; 32 / V lanes each l
      const uint32_t own = threadIdx.x % V, before = own + V < 2 * V - 1;
      for (uint32_t k0 = warp * 32; k0 < count; k0 += a.tables * 32) {
        const uint32_t k = k0 + threadIdx.x % 32, l = k / V;
        const float* at = sums + own * stride + l;
        float v = l < a.lanes ? at[0] : 0.0f;
        const bool other = l > 0 && l <= a.lanes && before;
        if (other) v += at[V * stride - 1];
        for (uint32_t w = 1; w < a.rows; ++w) {
          if (l < a.lanes) v += at[w * a.lanes];
          if (other) v += at[V * stride - 1 + w * a.lanes];
        }
        const int u = k < count ? ids[k] : -1;
        table_add(tables + warp * a.n_buckets, tags + warp * a.n_buckets, (uint32_t)u < a.n_buckets ? u : -1, v);
      }
    }
  }
  __syncthreads();
  write_partials(a, tables);
}

// As bias_fwd_few_kernel: a warp takes 32 neighbouring keys at a time, adds the samples up and the sums into its own table.  It is
// bound by the chain of that addition, eight times in a row: shuffles, tag, look whether it is still there, add, each waiting for the
// one before ([1, 16, 1024, 1024], 3969 buckets: 29 % of the issue slots, a warp waits 2.9 cycles for fixed latencies and 4.5 for memory, global and
// shared, to each instruction).  So as many warps run as have room for a table (asking for the next keys ahead of the additions:
// no gain).
template <int DT>
__global__ void __launch_bounds__(kFewThreads, kFewPerSm) bias_bwd_few_kernel(BiasArgs a) {
  using T = typename Io<DT>::T;
  extern __shared__ __align__(16) float sums[];  // [tables][n_buckets]; [tables][n_buckets] their tags
  enter_grid();
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, h = blockIdx.y;
  for (uint32_t i = threadIdx.x; i < a.tables * a.n_buckets; i += a.threads) sums[i] = 0.0f;
  __syncthreads();
  float* table = sums + warp * a.n_buckets;
  uint8_t* tags = (uint8_t*)(sums + a.tables * a.n_buckets) + warp * a.n_buckets;
  const uint64_t hop = (uint64_t)gridDim.x * a.tables * (32 * kFewKeys);
  for (uint64_t k0 = ((uint64_t)blockIdx.x * a.tables + warp) * (32 * kFewKeys); k0 < a.tk; k0 += hop) {
    const uint64_t k = k0 + lane;
    const int all = clamp_int((int64_t)(a.tk - k0)), left = all - (int)lane;
    const T* x = (const T*)a.x + h * a.slab + k;
    int u[kFewKeys];
    float v[kFewKeys];
#pragma unroll
    for (int i = 0; i < kFewKeys; ++i) {
      u[i] = i * 32 < left ? a.buckets[k + i * 32] : -1;
      v[i] = i * 32 < left ? Io<DT>::widen(x[i * 32]) : 0.0f;
    }
    for (uint32_t b = 1; b < a.batch; ++b) {
      x += a.sample;
#pragma unroll
      for (int i = 0; i < kFewKeys; ++i)
        if (i * 32 < left) v[i] += Io<DT>::widen(x[i * 32]);
    }
#pragma unroll
    for (int i = 0; i < kFewKeys; ++i)
      if (i * 32 < all) table_add(table, tags, (uint32_t)u[i] < a.n_buckets ? u[i] : -1, v[i]);
  }
  __syncthreads();
  write_partials(a, sums);
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

// What things cost a thread, in rows walked: an item; a slot whose bucket it looks up or adds; a run along the query rows, whose cut
// rows are a wait of their own.
struct Costs {
  uint32_t item, slot, run;
};
// Counting the slots makes chunks narrower and puts threads side by side along the batch: [64, 12, 197, 197] under a map backward
// 23.2 -> 19.3 us, forward 25.8 -> 25.0; [2, 16, 2048, 2048] backward 58 -> 53.  Counting the runs makes blocks taller: [16, 16, 577, 577]
// by distance backward 50 -> 41; forward does not gain by it (81 -> 88).
constexpr Costs kFwdCosts = {8, 1, 0}, kBwdCosts = {12, 2, 6};

// Cuts the work of every head into items: of the cuts tried, the one whose CTAs are done first, where every SM of a B200 holds
// kThreadsPerSm threads.  At most `most` CTAs over all heads.
template <int V>
void cut(BiasArgs& a, uint64_t most, const Costs& cost) {
  a.by_batch = a.tq < 4 * V;  // with few query rows the inner loop runs over the samples
  a.step = (uint32_t)((a.by_batch ? a.sample : a.tk + 1) % V);
  a.shift = 0;
  while ((1u << a.shift) < V && (a.step >> a.shift) % 2 == 0) ++a.shift;
  a.period = V >> a.shift;
  a.odd = a.step >> a.shift;
  a.period_log = (V == 8 ? 3 : 2) - a.shift;
  a.classes = a.tq == 1 ? a.period : V;
  uint64_t best = ~0ull;
  // heights of an item, in multiples of V
  for (uint32_t block = a.by_batch ? V : 32; block <= (a.by_batch ? (uint32_t)V : 256u); block += block < 128 ? 16 : 32) {
    const uint32_t height = block < a.tq ? block : a.tq;
    const uint64_t blocks = ceil_div(a.tq, height);
    const uint64_t vecs = (a.tk + V - 2) / V + 1 + (height + V - 2) / V;  // that the rows of a block can need, whatever their class
    for (uint32_t width : {kMostThreads, kThreads, 160u})
      for (uint32_t side = 1; side <= 16; side *= 2) {  // threads of a CTA; how many of them side by side along the batch
        if (side > 1 && width / side * 2 < 16) break;
        const uint64_t chunks = ceil_div(vecs, width / side);
        const uint32_t lanes = (uint32_t)ceil_div(vecs, chunks);
        // along the samples each row of threads has whole periods of them
        const uint32_t least = a.by_batch ? a.period : 1, fit = width / lanes, most_rows = (a.batch + least - 1) / least;
        const uint32_t rows = fit < most_rows ? fit : most_rows;
        const uint32_t share = rows * least, shares = (a.batch + share - 1) / share;  // samples that one row of every thread takes
        const uint32_t threads = (lanes * rows + 31) / 32 * 32;
        const uint64_t resident = 148u * (kThreadsPerSm / threads), ctas = resident < most ? resident : most;
        const uint64_t per_head = ctas > a.heads ? ctas / a.heads : 1;
        uint64_t parts = per_head / (blocks * chunks);
        parts = parts < 1 ? 1 : (parts < shares ? parts : shares);
        const uint32_t part = (uint32_t)((shares + parts - 1) / parts) * share;
        parts = (a.batch + part - 1) / part;
        const uint64_t items = blocks * chunks * parts;
        const uint64_t time = ((items + per_head - 1) / per_head) *
                              ((uint64_t)(height + (a.by_batch ? 0 : cost.run * a.period)) * (part / rows) + cost.item +
                               cost.slot * ((lanes * V + threads - 1) / threads));
        if (time >= best || items > 0xffffffffull) continue;
        best = time;
        a.block = height;
        a.lanes = lanes;
        a.rows = rows;
        a.threads = threads;
        a.chunks = (uint32_t)chunks;
        a.part = part;
        a.parts = (uint32_t)parts;
        a.items = (uint32_t)items;
        a.ctas_per_head = (uint32_t)(items < per_head ? items : per_head);
      }
    if (height == a.tq) break;
  }
  a.row_step = (int64_t)(a.by_batch ? (uint64_t)a.rows * a.period * a.sample : (uint64_t)a.period * (a.tk + 1));
  a.key_step = a.by_batch ? 0 : (int)a.period;
}

BiasArgs shape_args(uint32_t batch, uint32_t heads, uint32_t tq, uint32_t tk, uint32_t n_buckets, bool by_distance) {
  BiasArgs a = {};
  a.batch = batch;
  a.heads = heads;
  a.tq = by_distance ? tq : 1;
  a.tk = by_distance ? tk : (uint64_t)tq * tk;
  a.slab = (uint64_t)tq * tk;
  a.sample = a.slab * heads;
  a.n_buckets = n_buckets;
  return a;
}

// CTAs of the backward kernel, of which each writes a table: fewer for tables of many buckets.
uint64_t bwd_most(uint32_t n_buckets) {
  const uint64_t by_table = (1ull << 22) / n_buckets, most = 148 * 8;
  return by_table < most ? by_table : most;
}

template <int DT>
cudaError_t launch_bias_fwd(BiasArgs& a, cudaStream_t st) {
  constexpr int V = kVec<DT>;
  if (a.tq == 1 && a.batch <= kFewSamplesFwd) {
    const uint64_t resident = 148u * kFewPerSm, fit = resident > a.heads ? resident / a.heads : 1, want = ceil_div(a.tk, kFewKeys * kFewThreads);
    const uint64_t ctas = want < fit ? want : fit;
    a.column = a.n_buckets <= kColumnBuckets && a.tk >= (uint64_t)a.n_buckets * ctas;
    static_assert(kColumnBuckets * sizeof(float) <= 48 * 1024, "what a CTA has without asking");
    return launch_overlapped(bias_fwd_few_kernel<DT>, dim3((unsigned)ctas, a.heads), kFewThreads, a.column ? a.n_buckets * sizeof(float) : 0, st, a);
  }
  cut<V>(a, ~0ull, kFwdCosts);
  return launch_overlapped(bias_fwd_kernel<DT>, dim3(a.ctas_per_head, a.heads), a.threads, spread_slots<V>(a.lanes) * sizeof(float), st, a);
}

template <int DT>
cudaError_t launch_bias_bwd(BiasArgs& a, cudaStream_t st) {
  constexpr int V = kVec<DT>;
  static std::atomic<uint64_t> ready = {}, few_ready = {};
  const uint32_t few_tables = kFewTableBytes / (a.n_buckets * (uint32_t)(sizeof(float) + 1));
  if (a.tq == 1 && a.batch <= kFewSamplesBwd && few_tables >= 4) {
    a.tables = few_tables < kFewThreads / 32 ? few_tables : kFewThreads / 32;
    a.threads = a.tables * 32;
    const size_t smem = (size_t)a.tables * a.n_buckets * (sizeof(float) + 1);
    const uint64_t per_sm = few_tables / a.tables < kFewPerSm ? few_tables / a.tables : kFewPerSm;
    const uint64_t resident = 148 * per_sm, most = resident < bwd_most(a.n_buckets) ? resident : bwd_most(a.n_buckets);
    const uint64_t fit = most > a.heads ? most / a.heads : 1, want = ceil_div(a.tk, (uint64_t)a.threads * kFewKeys);
    a.ctas_per_head = (uint32_t)(want < fit ? want : fit);
    const cudaError_t e = allow_shared(bias_bwd_few_kernel<DT>, kFewTableBytes, few_ready);
    return e != cudaSuccess ? e : launch_overlapped(bias_bwd_few_kernel<DT>, dim3(a.ctas_per_head, a.heads), a.threads, smem, st, a);
  }
  cut<V>(a, bwd_most(a.n_buckets), kBwdCosts);
  const size_t count = slots<V>(a.lanes);
  // a table for each warp, unless they take too much shared memory, or a warp has less than two rows of slots to add
  const uint32_t room = (uint32_t)(kTableBytes / (a.n_buckets * (sizeof(float) + 1))), use = (uint32_t)(count / 64);
  a.tables = a.threads / 32 < room ? a.threads / 32 : room;
  a.tables = a.tables < use ? a.tables : use;
  if (a.tables < 1) a.tables = 1;
  const size_t smem = ((size_t)(a.threads + 32 / V) * (2 * V - 1) + (size_t)a.tables * a.n_buckets) * sizeof(float) + count * sizeof(int32_t) +
                      (size_t)a.tables * a.n_buckets;
  // the most that any shape takes: 189 KB
  constexpr size_t most = ((size_t)(kMostThreads + 32 / V) * (2 * V - 1) + kMaxBuckets) * sizeof(float) +
                          slots<V>(kMostThreads) * sizeof(int32_t) + kMaxBuckets;
  static_assert(most <= 227 * 1024, "a CTA must fit an SM");
  const cudaError_t e = allow_shared(bias_bwd_kernel<DT>, most, ready);
  return e != cudaSuccess ? e : launch_overlapped(bias_bwd_kernel<DT>, dim3(a.ctas_per_head, a.heads), a.threads, smem, st, a);
}

}  // namespace

uint64_t relbias_scratch_bytes(uint32_t heads, uint32_t n_buckets) {
  const uint64_t ctas = bwd_most(n_buckets);
  return (ctas > heads ? ctas : heads) * n_buckets * sizeof(float);
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

// A product of at most kMaxBuckets / 2 whole numbers below 2^32, exactly: words, low ones first.
struct WholeProduct {
  uint32_t words = 1, w[kMaxBuckets / 2];
  WholeProduct() { w[0] = 1; }
  void times(uint32_t f) {
    uint64_t carry = 0;
    for (uint32_t i = 0; i < words; ++i) {
      carry += (uint64_t)w[i] * f;
      w[i] = (uint32_t)carry;
      carry >>= 32;
    }
    if (carry) w[words++] = (uint32_t)carry;
  }
  bool at_least(const WholeProduct& o) const {
    if (words != o.words) return words > o.words;
    for (uint32_t i = words; i-- > 0;)
      if (w[i] != o.w[i]) return w[i] > o.w[i];
    return true;
  }
};

// Whether n >= e (m / e)^(j / w) for 0 < j < w: n^w >= e^(w - j) m^j, the fraction in lowest terms.
static bool reaches(uint32_t n, uint32_t e, uint32_t m, uint32_t j, uint32_t w) {
  const uint32_t f = (uint32_t)std::gcd(j, w);
  j /= f;
  w /= f;
  WholeProduct left, right;
  for (uint32_t i = 0; i < w; ++i) {
    left.times(n);
    right.times(i < j ? m : e);
  }
  return left.at_least(right);
}

// The bucket of a distance, on the host.  Buckets of short distances hold one distance each; past max_exact (half of a
// side's buckets) they widen geometrically up to max_distance: bucket max_exact + j starts at the smallest n with
// n >= max_exact (max_distance / max_exact)^(j / (side - max_exact)).  The power is taken in long double, off by less than 3e-18 of
// itself (a few roundings of 2^-64, of which that of the exponent counts up to 21 times).  Where a whole number is within 1e-17, whole
// numbers decide: borders that are whole themselves (8 * 16^(2/4) is 32), and those that lie just above one (with 256 buckets of
// one distance, 256 wide ones and max_distance 1,073,822,369, border 223 is 6e-8 above 150,392,436).
void log_buckets(int32_t* out, int64_t first, uint64_t count, uint32_t n_buckets, uint32_t max_distance, bool bidirectional) {
  const uint32_t side = bidirectional ? n_buckets / 2 : n_buckets, exact = side / 2, wide = side - exact;
  const auto start = [=](uint32_t u) -> int64_t {  // the smallest n of bucket u of a side; beyond the last, no end
    if (u <= exact) return u;
    if (u >= side) return INT64_MAX;
    const long double v = exact * powl((long double)max_distance / exact, (long double)(u - exact) / wide), near = roundl(v);
    if (fabsl(v - near) > 1e-17L * v) return (int64_t)ceill(v);
    return (int64_t)near + (reaches((uint32_t)near, exact, max_distance, u - exact, wide) ? 0 : 1);
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
