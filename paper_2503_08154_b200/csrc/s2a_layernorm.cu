// Layer norm forward and backward, with the gradients of its weights.
//
//   forward   mean = sum x / L, var = sum (x - mean)^2 / L, rstd = 1 / sqrt(var + eps),
//             y = (x - mean) rstd gamma + beta; (mean, rstd) of the row are kept, 8 bytes a row
//   backward  a = g gamma, xhat = (x - mean) rstd,
//             grad_in = rstd (a - sum a / L - xhat sum(a xhat) / L),
//             grad_gamma = sum over rows of g xhat, grad_beta = sum over rows of g
//
// Both passes are bound by memory: a row is read once and written once.  A row belongs to a team of LANES threads (8 to
// 512) that own NO * 8 elements each, in pieces of 16 bytes, and the next rows of a team are always on the way: every
// thread copies its own pieces into a ring of STAGES rows in shared memory (cp.async), so the bytes in flight do not cost
// registers, and since it reads back only what it copied itself the ring needs no barrier.  The variance is taken around
// the mean (no difference of squares); the warps of a row merge (count, mean, squared deviations) with one exchange (Chan,
// Golub and LeVeque's pairwise update).  All sums are binary32, but for those of rows beyond 16384 elements.
//
// Rows need not start on a 16-byte boundary.  A row's first element then sits s elements into a vector, pieces are the
// vectors of the memory (piece v holds V columns from V v - s on), and the two at the row's ends are masked (EDGE).  A team keeps
// to rows of one s, so that its pieces mean the same columns in every row.
//
// The weights' gradients are sums over rows: a thread keeps the sums of its own columns in registers over all the rows
// of its team, a CTA adds its teams' sums in order and writes one pair of rows to the caller's scratch, and a second kernel
// adds those in order: no atomics, the same bits on every run.
//
// What it measures on a B200 (6.57 TB/s copy rate): [12608, 768] bfloat16 forward 8.0 us (4.8 TB/s), backward with weights
// 14.6 us (4.0 TB/s), without 10.8 us (5.4 TB/s); of these about 2 us are the launch, 1.4 us the first rows' way from memory,
// and 3 us the second kernel of the weights' gradients.  [65536, 4096] backward 263 us (6.1 TB/s) in short runs, 291 to 307 us (5.2 to 5.5 TB/s) in
// long ones, where the clocks are lower.  The first kernels, with rows loaded into registers one at a time, took 17.3 us (forward) and 49.8 us
// (backward) on [12608, 768].  Rows off the 16-byte grid cost instructions, not bytes (half of the issue slots at 16 warps an SM): the masks of their ends
// are compared anew in every row, and one lane stores an end's elements one by one while its warp waits.  [4616, 1025] binary32 backward
// 16.8 us (3.4 TB/s), [20000, 1025] bfloat16 forward 30.6 us (2.7 TB/s).
#include "s2a_launch.h"
#include "s2a_oct.cuh"

namespace s2a {
namespace {

constexpr uint32_t kMaxPartials = 444;  // partial sums of the weights' gradients: three CTAs per SM of a B200

struct NormArgs {
  const void* x;
  const void* g;         // backward only
  const void* gamma;     // may be NULL (ones)
  const void* beta;      // forward only, may be NULL (zeros)
  void* out;             // y or grad_in
  const float* stats_in;
  float* stats_out;      // may be NULL
  float* partials;       // backward with weight gradients: [CTA][2][row_len]
  uint64_t n_rows;
  uint64_t x_stride, g_stride, out_stride;
  uint32_t row_len;
  int wdt;
  float eps;
  int g_apart, out_apart;  // EDGE: g's (out's) rows do not sit on the 16-byte grid as x's do: element by element
};

template <int DT, int NO> constexpr int kPieces = NO * 8 / kVec<DT>;  // pieces of a thread: NO * 8 elements

__host__ __device__ constexpr int threads_of(int lanes) { return lanes > 256 ? lanes : 256; }
// CTAs of the forward kernel on an SM.  Three of them hide the meeting of a row's warps better where their registers (80 a
// thread) suffice without spills: [65536, 4096] bfloat16 193 us against 199 with two and 242 with four; in binary32, with half
// the elements to a byte, two are ahead ([12608, 2048] 38.4 us against 39.7).  The widest teams, of 12289 elements on, spill (up to 172 bytes a
// thread off the grid, at the 128 registers that 512 threads leave): [8192, 16384] bfloat16 91 us (5.9 TB/s), [8192, 16383] 292 us (1.8 TB/s).
__host__ __device__ constexpr int fwd_ctas(int dt, bool edge, int no, int lanes) {
  return lanes > 256 ? 1 : (no == 1 ? 4 : (no == 2 && dt == kBF16 && !edge ? 3 : 2));
}
// And of the backward kernel: three for short rows ([300000, 64] bfloat16 23.4 us against 32 with two), two for longer ones
// ([65536, 4096] 263 us against 281 with three).
__host__ __device__ constexpr int bwd_ctas(bool edge, int no, int lanes) { return lanes > 256 ? 1 : (no == 1 && !edge ? 3 : 2); }
// Rows in flight per team: what keeps two CTAs of an SM (one of 512 threads) within its shared memory.
__host__ __device__ constexpr int stages_of(int stage_bytes) {
  return stage_bytes <= 24 * 1024 ? 4 : (stage_bytes <= 32 * 1024 ? 3 : (stage_bytes <= 100 * 1024 ? 2 : 1));
}
__host__ __device__ constexpr int stage_bytes(int dt, int no, int lanes, int tensors) {
  return threads_of(lanes) * no * (dt == kF32 ? 32 : 16) * tensors + (tensors == 2 ? threads_of(lanes) * 8 : 0);
}

// Where a thread's pieces lie: piece j begins at column (j * LANES + lane) * kVec - s (s = 0 without EDGE).
template <int DT, int LANES>
__device__ __forceinline__ int piece_column(int j, uint32_t lane, int s) { return (int)((j * LANES + lane) * (uint32_t)kVec<DT>) - s; }

// A team is the smallest that holds the row, so the row's last vector lies in one of a thread's last two pieces (three of the
// shorter ones of binary32): only from piece kSure on may a piece end after the row, or begin after it.
template <int DT, int NO> constexpr int kSure = kPieces<DT, NO> - (DT == kF32 ? 3 : 2);

template <int DT>
__device__ __forceinline__ bool piece_whole(int c, int L) { return c >= 0 && c + kVec<DT> <= L; }

// Starts the copies of a row's pieces into this thread's column of a stage, [piece][thread] of 16 bytes.  Elements after the row's end
// come out as zeros; the elements before its beginning that share its first vector are another row's, and cut_head clears
// them.  Where the tensor itself begins inside that vector, and in a tensor that sits on another grid (`apart`), pieces are read
// element by element.
template <int DT, bool EDGE, int NO, int LANES, int THREADS>
__device__ __forceinline__ void fetch(uint4* slot, const void* tensor, uint64_t row, uint64_t stride, uint32_t lane, int L, int s,
                                      bool apart) {
  using T = typename Io<DT>::T;
  constexpr int V = kVec<DT>;
  const T* p = (const T*)tensor + row * stride;
#pragma unroll
  for (int j = 0; j < kPieces<DT, NO>; ++j) {
    const int c = piece_column<DT, LANES>(j, lane, s);
    const bool sure = j < kSure<DT, NO>;
    if (!sure && c >= L) continue;
    if (!EDGE || (sure && j > 0 && !apart)) {
      copy_async<16>(slot + j * THREADS, p + c);
    } else if (!apart && (j > 0 || p + c >= (const T*)tensor)) {
      copy_async_front(slot + j * THREADS, p + c, min(L - c, V) * (int)sizeof(T));
    } else {
      float f[V];
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = c + i >= 0 && c + i < L ? Io<DT>::widen(p[c + i]) : 0.0f;
      F2 w[V / 2];
#pragma unroll
      for (int i = 0; i < V / 2; ++i) w[i] = f2_pack(f[2 * i], f[2 * i + 1]);
      slot[j * THREADS] = narrow_piece<DT>(w);
    }
  }
}

// What a thread's first piece keeps of its 16 bytes: all of it but for the first s elements of a row's first vector.
template <int DT>
__device__ __forceinline__ uint4 head_mask(uint32_t lane, int s) {
  uint32_t m[4] = {~0u, ~0u, ~0u, ~0u};
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < kVec<DT>; ++i)
      if (i < s) m[DT == kF32 ? i : i / 2] &= DT == kF32 ? 0u : (i % 2 ? 0x0000ffffu : 0xffff0000u);
  return make_uint4(m[0], m[1], m[2], m[3]);
}
template <int DT, bool EDGE>
__device__ __forceinline__ uint4 cut_head(uint4 r, int j, const uint4& mask) {
  if (EDGE && j == 0) {
    r.x &= mask.x;
    r.y &= mask.y;
    r.z &= mask.z;
    r.w &= mask.w;
  }
  return r;
}

// Elements of a piece outside the row become zero.
template <int DT>
__device__ __forceinline__ void mask_ends(F2* v, int c, int L) {
  if (piece_whole<DT>(c, L)) return;
#pragma unroll
  for (int i = 0; i < kPairs<DT>; ++i) {
    float lo, hi;
    f2_unpack(v[i], lo, hi);
    const int k = c + 2 * i;
    v[i] = f2_pack(k >= 0 && k < L ? lo : 0.0f, k + 1 >= 0 && k + 1 < L ? hi : 0.0f);
  }
}

template <int DT, bool EDGE>
__device__ __forceinline__ void put_piece(typename Io<DT>::T* row, int c, int L, bool whole, bool apart, const F2* v) {
  if (!EDGE || (!apart && (whole || piece_whole<DT>(c, L)))) {
    *(uint4*)(row + c) = narrow_piece<DT>(v);
  } else {
#pragma unroll
    for (int i = 0; i < kVec<DT>; ++i) {
      float lo, hi;
      f2_unpack(v[i / 2], lo, hi);
      if (c + i >= 0 && c + i < L) row[c + i] = Io<DT>::narrow(i % 2 ? hi : lo);
    }
  }
}

// A piece's learned parameters, from column c on; `fill` where there are none.
template <int DT>
__device__ __forceinline__ void load_weights(const void* p, int c, int L, int wdt, float fill, F2* v) {
  constexpr int V = kVec<DT>;
  if (p && piece_whole<DT>(c, L)) {
    const char* at = (const char*)p + (int64_t)c * (wdt == kF32 ? 4 : 2);
    if (wdt == kF32 && ((uintptr_t)at & 15u) == 0) {
#pragma unroll
      for (int i = 0; i < V / 4; ++i) widen_piece<kF32>(((const uint4*)at)[i], v + 2 * i);
      return;
    }
    if (wdt == kBF16 && ((uintptr_t)at & (2 * V - 1)) == 0) {
      const uint2 a = *(const uint2*)at, b = V == 8 ? ((const uint2*)at)[1] : a;
      v[0] = f2_from_bf16x2(a.x);
      v[1] = f2_from_bf16x2(a.y);
      if (V == 8) {
        v[V / 2 - 2] = f2_from_bf16x2(b.x);
        v[V / 2 - 1] = f2_from_bf16x2(b.y);
      }
      return;
    }
  }
  float f[V];
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = p && c + i >= 0 && c + i < L ? load_param(p, (uint64_t)(c + i), wdt) : fill;
#pragma unroll
  for (int i = 0; i < V / 2; ++i) v[i] = f2_pack(f[2 * i], f[2 * i + 1]);
}

// A thread holds the weights of its columns in registers for all its rows (read from shared memory in every row instead, they cost
// more than the occupancy gives: 10.5 us at four CTAs an SM against 8.1 on [12608, 768]).
// Where several teams share a CTA, its weights come through shared memory, each loaded once for all teams.  The loads are
// sent out before the rows' copies: behind those they take as long as the whole first filling of the ring (5.4 us instead
// of about 1 on [12608, 768]).
template <int LANES> constexpr bool kStaged = LANES <= 64;
template <int NO, int LANES> constexpr int kStagedFloats = kStaged<LANES> ? NO * 8 * LANES : 0;
template <int NO, int LANES>
struct Staged {
  static constexpr int kEach = NO * 8 * LANES / threads_of(LANES) > 0 ? NO * 8 * LANES / threads_of(LANES) : 1;
  float v[kEach];
  __device__ __forceinline__ void load(const void* p, int L, int wdt, float fill) {
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int c = k * threads_of(LANES) + (int)threadIdx.x;
      v[k] = p && c < L ? load_param(p, (uint64_t)c, wdt) : fill;
    }
  }
  __device__ __forceinline__ void put(float* row, int L) const {
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int c = k * threads_of(LANES) + (int)threadIdx.x;
      if (c < L) row[c] = v[k];
    }
  }
};
// A piece of a staged row.
template <int DT, bool EDGE>
__device__ __forceinline__ void take_piece(const float* row, int c, int L, F2* v) {
  if (!EDGE) {
#pragma unroll
    for (int i = 0; i < kVec<DT> / 4; ++i) {
      const float4 w = c < L ? ((const float4*)(row + c))[i] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      v[2 * i] = f2_pack(w.x, w.y);
      v[2 * i + 1] = f2_pack(w.z, w.w);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPairs<DT>; ++i) {
      const int k = c + 2 * i;
      v[i] = f2_pack(k >= 0 && k < L ? row[k] : 0.0f, k + 1 >= 0 && k + 1 < L ? row[k + 1] : 0.0f);
    }
  }
}

__device__ __forceinline__ float f2_sum(F2 a) {
  float lo, hi;
  f2_unpack(a, lo, hi);
  return lo + hi;
}

// Sum over the lanes of a team that lie in one warp (or over groups of W lanes).
template <int W>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// sum / count, given 1 / count.  For bfloat16 rows what the product lacks of the sum is added, which makes the mean of a row of one
// value that value (the sum of up to 16384 of 8 bits each is exact, and so is the quotient).  Binary32 rows have a rule of their own.
template <int DT>
__device__ __forceinline__ float mean_of(float sum, float count, float inv_count) {
  const float q = sum * inv_count;
  if (DT == kF32) return q;
  const float whole = fmaf(fmaf(-q, count, sum), inv_count, q);
  return whole == whole ? whole : q;  // an infinite sum leaves no remainder
}

template <int LANES>
__device__ __forceinline__ void team_barrier(uint32_t team) {
  if (LANES > 32) asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(LANES) : "memory");
}

// The shift s of a row: how many elements of its first vector lie before it.
template <int DT, bool EDGE>
__device__ __forceinline__ int row_shift(const NormArgs& a, uint64_t row) {
  using T = typename Io<DT>::T;
  return EDGE ? (int)((((uintptr_t)a.x / sizeof(T)) + row * a.x_stride) % kVec<DT>) : 0;
}

// ---------------------------------------------------------------- forward
template <int DT, bool EDGE, int NO, int LANES>
__global__ void __launch_bounds__(threads_of(LANES), fwd_ctas(DT, EDGE, NO, LANES)) norm_fwd_kernel(NormArgs a) {
  using T = typename Io<DT>::T;
  constexpr int THREADS = threads_of(LANES), TEAMS = THREADS / LANES, WARPS = LANES / 32 > 1 ? LANES / 32 : 1;
  constexpr int GROUP = LANES < 32 ? LANES : 32;
  constexpr int BYTES = stage_bytes(DT, NO, LANES, 1), STAGES = stages_of(BYTES);
  extern __shared__ __align__(16) char ring[];
  __shared__ float4 merge[2][TEAMS][WARPS];  // (mean, deviations, count) of each warp of a row, two rows' worth
  enter_grid();
  const uint32_t team = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const int L = (int)a.row_len;
  const float inv_l = 1.0f / (float)L;
  const uint64_t step = (uint64_t)gridDim.x * TEAMS, first = (uint64_t)blockIdx.x * TEAMS + team;
  const int s = row_shift<DT, EDGE>(a, first);
  const uint4 head = head_mask<DT>(lane, s);
  constexpr int NP = kPieces<DT, NO>, PAIRS = kPairs<DT>;
  Staged<NO, LANES> sg, sb;
  if (kStaged<LANES>) {
    sg.load(a.gamma, L, a.wdt, 1.0f);
    sb.load(a.beta, L, a.wdt, 0.0f);
  }
#pragma unroll
  for (int k = 0; k < STAGES; ++k) {
    if (first + k * step < a.n_rows)
      fetch<DT, EDGE, NO, LANES, THREADS>((uint4*)(ring + k * BYTES) + threadIdx.x, a.x, first + k * step, a.x_stride, lane, L, s, false);
    copy_commit();
  }
  float *gamma_row = (float*)(ring + STAGES * BYTES), *beta_row = gamma_row + kStagedFloats<NO, LANES>;
  if (kStaged<LANES>) {
    sg.put(gamma_row, L);
    sb.put(beta_row, L);
    __syncthreads();
  }
  F2 gamma[NP][PAIRS], beta[NP][PAIRS];
  float count = 0.0f;  // elements of the row that this warp holds
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    const int c = piece_column<DT, LANES>(j, lane, s);
    if (kStaged<LANES>) {
      take_piece<DT, EDGE>(gamma_row, c, L, gamma[j]);
      take_piece<DT, EDGE>(beta_row, c, L, beta[j]);
    } else {
      load_weights<DT>(a.gamma, c, L, a.wdt, 1.0f, gamma[j]);
      load_weights<DT>(a.beta, c, L, a.wdt, 0.0f, beta[j]);
    }
    if (c < L) count += (float)(min(c + kVec<DT>, L) - max(c, 0));
  }
  if (WARPS > 1) count = lanes_sum<32>(count);
  const float inv_count = WARPS > 1 ? (count > 0.0f ? 1.0f / count : 0.0f) : inv_l;
  uint32_t parity = 0, stage = 0;
  // the lanes of a warp that serve several rows keep together: a row past the end is computed on whatever the ring holds
  // and written nowhere
  for (uint64_t base = (uint64_t)blockIdx.x * TEAMS; base < a.n_rows; base += step) {
    const uint64_t r = base + team;
    if (LANES >= 32 && r >= a.n_rows) break;
    copy_wait<STAGES - 1>();
    uint4* slot = (uint4*)(ring + stage * BYTES) + threadIdx.x;
    F2 v[NP][PAIRS], sum = f2_both(0.0f);
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int c = piece_column<DT, LANES>(j, lane, s);
      if (j < kSure<DT, NO> || c < L) {
        widen_piece<DT>(cut_head<DT, EDGE>(slot[j * THREADS], j, head), v[j]);
      } else {
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) v[j][i] = f2_both(0.0f);
      }
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) sum = f2_add(sum, v[j][i]);
    }
    if (r + STAGES * step < a.n_rows)
      fetch<DT, EDGE, NO, LANES, THREADS>(slot, a.x, r + STAGES * step, a.x_stride, lane, L, s, false);
    copy_commit();
    stage = stage + 1 == STAGES ? 0 : stage + 1;
    float mean = mean_of<DT>(lanes_sum<GROUP>(f2_sum(sum)), WARPS > 1 ? count : (float)L, inv_count), dev;
    // v - by, and the sum of its squares over the lanes of a warp
    const auto centre = [&](float by) {
      F2 sq = f2_both(0.0f);
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        const int c = piece_column<DT, LANES>(j, lane, s);
        if (j >= kSure<DT, NO> && c >= L) continue;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) v[j][i] = f2_sub(v[j][i], f2_both(by));
        if (EDGE && (j == 0 || j >= kSure<DT, NO>)) mask_ends<DT>(v[j], c, L);  // elements outside the row have no deviation
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) sq = f2_fma(v[j][i], v[j][i], sq);
      }
      return lanes_sum<GROUP>(f2_sum(sq));
    };
    dev = centre(mean);
    if (WARPS > 1) {
      if (lane % 32 == 0) merge[parity][team][lane / 32] = make_float4(mean, dev, count, 0.0f);
      // the two buffers alternate: a warp writes one of them again only after the next barrier (of the next row, or below), which
      // every warp of the team reaches after it has read this row's values
      team_barrier<LANES>(team);
      const float4 m = merge[parity][team][lane % WARPS];
      float shift = mean;  // from x - mean of the warp to x - mean
      mean = mean_of<DT>(lanes_sum<WARPS>(m.z * m.x), (float)L, inv_l);
      shift -= mean;
      dev = lanes_sum<WARPS>(m.y + m.z * (m.x - mean) * (m.x - mean));
      parity ^= 1;
#pragma unroll
      for (int j = 0; j < NP; ++j)
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) v[j][i] = f2_add(v[j][i], f2_both(shift));
    }
    // A binary32 row whose mean is large beside its spread, 64 times or more: the mean's rounding, no longer small beside the spread
    // (and all there is, in a row of one value), is the mean of the deviations from it, and is taken out of them.  bfloat16 rows
    // need it not (mean_of; and two neighbouring values are 2^-8 apart).  It costs the binary32 rows some 3 %.
    const bool far = dev * inv_l + a.eps < mean * mean * 0x1p-12f;
    if (DT == kF32 && __builtin_expect(LANES < 32 ? __any_sync(0xffffffffu, far) != 0 : far, 0)) {
      const auto team_sum = [&](float t) {  // of the warps' sums
        if (WARPS > 1) {
          if (lane % 32 == 0) merge[parity][team][lane / 32].x = t;
          team_barrier<LANES>(team);
          t = lanes_sum<WARPS>(merge[parity][team][lane % WARPS].x);
          parity ^= 1;
        }
        return t;
      };
      F2 rest = f2_both(0.0f);
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        const int c = piece_column<DT, LANES>(j, lane, s);
        if (j >= kSure<DT, NO> && c >= L) continue;
        if (EDGE && WARPS > 1 && (j == 0 || j >= kSure<DT, NO>)) mask_ends<DT>(v[j], c, L);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) rest = f2_add(rest, v[j][i]);
      }
      float lean = team_sum(lanes_sum<GROUP>(f2_sum(rest))) * inv_l;
      if (!far) lean = 0.0f;  // another row of the warp: this one keeps its bits
      dev = team_sum(centre(lean));
      mean += lean;
    }
    const float rstd = __frsqrt_rn(dev * inv_l + a.eps);
    if (LANES < 32 && r >= a.n_rows) continue;
    if (a.stats_out && lane == 0) ((float2*)a.stats_out)[r] = make_float2(mean, rstd);
    T* out = (T*)a.out + r * a.out_stride;
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int c = piece_column<DT, LANES>(j, lane, s);
      if (j >= kSure<DT, NO> && c >= L) continue;
#pragma unroll
      for (int i = 0; i < PAIRS; ++i)
        v[j][i] = f2_fma(f2_mul(v[j][i], f2_both(rstd)), gamma[j][i], beta[j][i]);
      put_piece<DT, EDGE>(out, c, L, j > 0 && j < kSure<DT, NO>, EDGE && a.out_apart, v[j]);
    }
  }
}

// ---------------------------------------------------------------- backward
template <int DT, bool EDGE, int NO, int LANES, bool WG>
__global__ void __launch_bounds__(threads_of(LANES), bwd_ctas(EDGE, NO, LANES)) norm_bwd_kernel(NormArgs a) {
  using T = typename Io<DT>::T;
  constexpr int THREADS = threads_of(LANES), TEAMS = THREADS / LANES, WARPS = LANES / 32 > 1 ? LANES / 32 : 1;
  constexpr int GROUP = LANES < 32 ? LANES : 32;
  constexpr int BYTES = stage_bytes(DT, NO, LANES, 2), STAGES = stages_of(BYTES);
  constexpr int NP = kPieces<DT, NO>, PAIRS = kPairs<DT>, TENSOR = NP * THREADS * 16;
  extern __shared__ __align__(16) char ring[];  // per stage: x's pieces, g's pieces, (mean, rstd) per thread
  __shared__ float2 merge[2][TEAMS][WARPS];
  enter_grid();
  const uint32_t team = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const int L = (int)a.row_len;
  const float inv_l = 1.0f / (float)L;
  const uint64_t step = (uint64_t)gridDim.x * TEAMS, first = (uint64_t)blockIdx.x * TEAMS + team;
  const int s = row_shift<DT, EDGE>(a, first);
  const uint4 head = head_mask<DT>(lane, s);
  const auto start_row = [&](char* at, uint64_t r) {
    if (r >= a.n_rows) return;
    fetch<DT, EDGE, NO, LANES, THREADS>((uint4*)at + threadIdx.x, a.x, r, a.x_stride, lane, L, s, false);
    fetch<DT, EDGE, NO, LANES, THREADS>((uint4*)(at + TENSOR) + threadIdx.x, a.g, r, a.g_stride, lane, L, s, EDGE && a.g_apart);
    copy_async<8>(at + 2 * TENSOR + threadIdx.x * 8, a.stats_in + 2 * r);
  };
  Staged<NO, LANES> staged;
  if (kStaged<LANES>) staged.load(a.gamma, L, a.wdt, 1.0f);
#pragma unroll
  for (int k = 0; k < STAGES; ++k) {
    start_row(ring + k * BYTES, first + k * step);
    copy_commit();
  }
  float* gamma_row = (float*)(ring + STAGES * BYTES);
  if (kStaged<LANES>) {
    staged.put(gamma_row, L);
    __syncthreads();
  }
  F2 gamma[NP][PAIRS], dgamma[NP][PAIRS], dbeta[NP][PAIRS];
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    const int c = piece_column<DT, LANES>(j, lane, s);
    if (kStaged<LANES>) take_piece<DT, EDGE>(gamma_row, c, L, gamma[j]);
    else load_weights<DT>(a.gamma, c, L, a.wdt, 1.0f, gamma[j]);
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) dgamma[j][i] = dbeta[j][i] = f2_both(0.0f);
  }
  uint32_t parity = 0, stage = 0;
  for (uint64_t base = (uint64_t)blockIdx.x * TEAMS; base < a.n_rows; base += step) {
    const uint64_t r = base + team;
    if (LANES >= 32 && r >= a.n_rows) break;  // narrower teams share a warp and keep together
    const bool on = LANES >= 32 || r < a.n_rows;
    copy_wait<STAGES - 1>();
    char* at = ring + stage * BYTES;
    const uint4 *sx = (const uint4*)at + threadIdx.x, *sg = (const uint4*)(at + TENSOR) + threadIdx.x;
    const float2 st = *(const float2*)(at + 2 * TENSOR + threadIdx.x * 8);
    const F2 mean2 = f2_both(st.x), rstd2 = f2_both(st.y);
    F2 s1 = f2_both(0.0f), s2 = f2_both(0.0f);
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int c = piece_column<DT, LANES>(j, lane, s);
      if (!on || (j >= kSure<DT, NO> && c >= L)) continue;
      F2 x[PAIRS], g[PAIRS];
      widen_piece<DT>(cut_head<DT, EDGE>(sx[j * THREADS], j, head), x);
      widen_piece<DT>(cut_head<DT, EDGE>(sg[j * THREADS], j, head), g);
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) {
        const F2 xc = f2_sub(x[i], mean2), w = f2_mul(g[i], gamma[j][i]);
        s1 = f2_add(s1, w);
        s2 = f2_fma(w, xc, s2);
        if (WG) {
          dgamma[j][i] = f2_fma(f2_mul(g[i], rstd2), xc, dgamma[j][i]);
          dbeta[j][i] = f2_add(dbeta[j][i], g[i]);
        }
      }
    }
    float c1 = lanes_sum<GROUP>(f2_sum(s1)), c2 = lanes_sum<GROUP>(f2_sum(s2));
    if (WARPS > 1) {
      if (lane % 32 == 0) merge[parity][team][lane / 32] = make_float2(c1, c2);
      team_barrier<LANES>(team);  // alternating buffers, as in the forward kernel
      const float2 m = merge[parity][team][lane % WARPS];
      c1 = lanes_sum<WARPS>(m.x);
      c2 = lanes_sum<WARPS>(m.y);
      parity ^= 1;
    }
    // with w = g gamma and xc = x - mean: grad_in = rstd w - rstd sum w / L - xc rstd^3 sum(w xc) / L
    const F2 k1 = f2_both(-st.y * (c1 * inv_l)), k2 = f2_both(-(st.y * (c2 * inv_l)) * st.y * st.y);
    T* out = (T*)a.out + r * a.out_stride;
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const int c = piece_column<DT, LANES>(j, lane, s);
      if (!on || (j >= kSure<DT, NO> && c >= L)) continue;
      F2 x[PAIRS], g[PAIRS];
      widen_piece<DT>(sx[j * THREADS], x);
      widen_piece<DT>(sg[j * THREADS], g);
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) {
        g[i] = f2_fma(f2_mul(g[i], gamma[j][i]), rstd2, f2_fma(f2_sub(x[i], mean2), k2, k1));
      }
      put_piece<DT, EDGE>(out, c, L, j > 0 && j < kSure<DT, NO>, EDGE && a.out_apart, g);
    }
    start_row(at, r + STAGES * step);
    copy_commit();
    stage = stage + 1 == STAGES ? 0 : stage + 1;
  }
  if constexpr (WG) {
    // The CTA's teams, column by column, in order.  The ring holds their sums by piece: [team][2][quarter][piece][lane] of four
    // columns, which threads write and read without bank conflicts.
    copy_wait<0>();
    __syncthreads();
    float4* sums = (float4*)ring;
    constexpr int QUADS = kVec<DT> / 4, kRow = QUADS * NP * LANES;  // float4s of a piece; of one of a team's two rows
#pragma unroll
    for (int j = 0; j < NP; ++j)
#pragma unroll
      for (int q = 0; q < QUADS; ++q) {
        float4 w;
        f2_unpack(dgamma[j][2 * q], w.x, w.y);
        f2_unpack(dgamma[j][2 * q + 1], w.z, w.w);
        sums[(team * 2 + 0) * kRow + (q * NP + j) * LANES + lane] = w;
        f2_unpack(dbeta[j][2 * q], w.x, w.y);
        f2_unpack(dbeta[j][2 * q + 1], w.z, w.w);
        sums[(team * 2 + 1) * kRow + (q * NP + j) * LANES + lane] = w;
      }
    __syncthreads();
    float* part = a.partials + (uint64_t)blockIdx.x * 2 * L;
    const float* flat = (const float*)ring;
    for (uint32_t k = threadIdx.x; k < 2u * (uint32_t)L; k += THREADS) {
      const uint32_t which = k >= (uint32_t)L, c = which ? k - L : k;
      float t = 0.0f;
      const auto at = [&](uint32_t p) { return flat + (which * kRow + ((p / 4) % QUADS) * NP * LANES + p / kVec<DT>) * 4 + p % 4; };
      const float* column = at(c);
#pragma unroll 8
      for (int m = 0; m < TEAMS; ++m) {
        if (EDGE) column = at(c + (uint32_t)row_shift<DT, EDGE>(a, (uint64_t)blockIdx.x * TEAMS + m));
        t += column[m * 2 * kRow * 4];
      }
      part[k] = t;
    }
  }
}

// Adds the partial rows: [n_part][2][row_len] -> grad_gamma, grad_beta (either may be NULL).  A CTA owns 32 columns
// of one of the two; its warps take every 32nd partial, all loads of a thread at once.  (CTAs of 128 threads that fit beside
// the main kernel's, with 8 columns each, take 1.6 us longer on [12608, 768].)
constexpr int kReduceWarps = 32;
__global__ void __launch_bounds__(kReduceWarps * 32) norm_reduce_kernel(const float* partials, uint32_t n_part, uint32_t L,
                                                                        void* dgamma, void* dbeta, int wdt) {
  __shared__ float sums[kReduceWarps][33];
  enter_grid();
  const uint32_t which = blockIdx.y, w = threadIdx.x / 32, c = blockIdx.x * 32 + threadIdx.x % 32;
  float acc = 0.0f;
  if (c < L) {
    const float* p = partials + (uint64_t)which * L + c;
    float v[kMaxPartials / kReduceWarps + 1];
#pragma unroll
    for (int k = 0; k <= kMaxPartials / kReduceWarps; ++k) {
      const uint32_t at = w + k * kReduceWarps;
      v[k] = at < n_part ? p[(uint64_t)at * 2 * L] : 0.0f;
    }
#pragma unroll
    for (int k = 0; k <= kMaxPartials / kReduceWarps; ++k) acc += v[k];
  }
  sums[w][threadIdx.x % 32] = acc;
  __syncthreads();
  // warp w adds up column w: lane k holds the sum of warp k
  acc = warp_sum(sums[threadIdx.x % 32][w]);
  void* out = which ? dbeta : dgamma;
  const uint32_t mine = blockIdx.x * 32 + w;
  if (threadIdx.x % 32 == 0 && mine < L && out) store_param(out, mine, wdt, acc);
}

// ---------------------------------------------------------------- rows too long for registers
// A CTA of 512 threads walks a row three times (sum; squared deviations; output), element by element.  A thread may have four million
// terms of a row: their sums are held in 64 bits, as terms that are alike would all be rounded the same way in 32 (30,000,001
// bfloat16 elements about 1.1: the variance was off by 1.6e-4 of itself).  Four CTAs on an SM in forward: [2048, 20000] bfloat16 87 us
// (1.9 TB/s) against 115 with three (40 registers a thread); backward is as fast with three where the rows are few
// ([64, 65537] 39 us against 43), 130 us (1.9 TB/s) on [2048, 20000], 240 us with the weights' gradients.  The loads are single
// elements, and a row comes from L2 in all passes but the first.
constexpr int kLongThreads = 512;

__device__ __forceinline__ double cta_sum(double v, double* buf) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if (threadIdx.x % 32 == 0) buf[threadIdx.x / 32] = v;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int w = 0; w < kLongThreads / 32; ++w) t += buf[w];
  return t;
}

template <int DT>
__global__ void __launch_bounds__(kLongThreads, 4) norm_fwd_long_kernel(NormArgs a) {
  using T = typename Io<DT>::T;
  __shared__ double buf[kLongThreads / 32];
  enter_grid();
  const uint32_t L = a.row_len;
  for (uint64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
    const T* x = (const T*)a.x + r * a.x_stride;
    T* y = (T*)a.out + r * a.out_stride;
    double s = 0.0;
    for (uint32_t c = threadIdx.x; c < L; c += kLongThreads) s += Io<DT>::widen(x[c]);
    const double exact = cta_sum(s, buf) / L;
    const float mean = (float)exact, lean = (float)(exact - mean);  // NaN where the mean is infinite, as x - mean is
    s = 0.0;
    for (uint32_t c = threadIdx.x; c < L; c += kLongThreads) {
      const float d = Io<DT>::widen(x[c]) - mean;
      s += d * d;
    }
    const float rstd = __frsqrt_rn((float)(cta_sum(s, buf) / L - (double)lean * lean) + a.eps);
    if (a.stats_out && threadIdx.x == 0) ((float2*)a.stats_out)[r] = make_float2(mean, rstd);
    for (uint32_t c = threadIdx.x; c < L; c += kLongThreads) {
      const float gm = a.gamma ? load_param(a.gamma, c, a.wdt) : 1.0f, bt = a.beta ? load_param(a.beta, c, a.wdt) : 0.0f;
      y[c] = Io<DT>::narrow(fmaf(((Io<DT>::widen(x[c]) - mean) - lean) * rstd, gm, bt));
    }
  }
}

template <int DT>
__global__ void __launch_bounds__(kLongThreads) norm_bwd_long_kernel(NormArgs a) {
  using T = typename Io<DT>::T;
  __shared__ double buf[kLongThreads / 32];
  enter_grid();
  const uint32_t L = a.row_len;
  for (uint64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
    const T* x = (const T*)a.x + r * a.x_stride;
    const T* g = (const T*)a.g + r * a.g_stride;
    T* out = (T*)a.out + r * a.out_stride;
    const float2 st = ((const float2*)a.stats_in)[r];
    double s1 = 0.0, s2 = 0.0;
    for (uint32_t c = threadIdx.x; c < L; c += kLongThreads) {
      const float w = Io<DT>::widen(g[c]) * (a.gamma ? load_param(a.gamma, c, a.wdt) : 1.0f);
      s1 += w;
      s2 += w * (Io<DT>::widen(x[c]) - st.x);
    }
    const float m1 = (float)(cta_sum(s1, buf) / L), m2 = (float)(cta_sum(s2, buf) * st.y / L);
    for (uint32_t c = threadIdx.x; c < L; c += kLongThreads) {
      const float w = Io<DT>::widen(g[c]) * (a.gamma ? load_param(a.gamma, c, a.wdt) : 1.0f);
      const float xhat = (Io<DT>::widen(x[c]) - st.x) * st.y;
      out[c] = Io<DT>::narrow((w - m1 - xhat * m2) * st.y);
    }
  }
}

// The weights' gradients of long rows: a thread owns one column and every gridDim.y-th row.  It runs before
// norm_bwd_long_kernel, whose output may take the place of g or x.
template <int DT>
__global__ void __launch_bounds__(256) norm_columns_long_kernel(NormArgs a) {
  using T = typename Io<DT>::T;
  enter_grid();
  const uint64_t c = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= a.row_len) return;
  float dg = 0.0f, db = 0.0f;
  for (uint64_t r = blockIdx.y; r < a.n_rows; r += gridDim.y) {
    const float2 st = ((const float2*)a.stats_in)[r];
    const float g = Io<DT>::widen(((const T*)a.g)[r * a.g_stride + c]), x = Io<DT>::widen(((const T*)a.x)[r * a.x_stride + c]);
    dg = fmaf(g, (x - st.x) * st.y, dg);
    db += g;
  }
  float* part = a.partials + (uint64_t)blockIdx.y * 2 * a.row_len;
  part[c] = dg;
  part[a.row_len + c] = db;
}

// ---------------------------------------------------------------- host side
uint64_t gcd64(uint64_t a, uint64_t b) {
  while (b) {
    const uint64_t t = a % b;
    a = b;
    b = t;
  }
  return a;
}

uint32_t partial_cap(uint64_t n_rows) { return (uint32_t)(n_rows < 1 ? 1 : (n_rows < kMaxPartials ? n_rows : kMaxPartials)); }

template <int DT, bool EDGE, int NO, int LANES>
cudaError_t launch_norm(bool fwd, bool wg, const NormArgs& a, uint32_t& parts, cudaStream_t st) {
  static std::atomic<uint64_t> ready[3] = {};
  constexpr int THREADS = threads_of(LANES), TEAMS = THREADS / LANES;
  constexpr int B1 = stage_bytes(DT, NO, LANES, 1), B2 = stage_bytes(DT, NO, LANES, 2);
  constexpr size_t weights = kStagedFloats<NO, LANES> * sizeof(float);  // a row of them
  constexpr size_t ring_fwd = (size_t)B1 * stages_of(B1) + 2 * weights, ring_bwd = (size_t)B2 * stages_of(B2) + weights;
  constexpr size_t sums = (size_t)THREADS * NO * 64;  // the teams' column sums take the ring's place
  constexpr size_t smem_wg = ring_bwd > sums ? ring_bwd : sums;
  const uint64_t want = (a.n_rows + TEAMS - 1) / TEAMS;
  const uint64_t per_sm = fwd ? fwd_ctas(DT, EDGE, NO, LANES) : bwd_ctas(EDGE, NO, LANES);
  uint64_t cap = fwd || !wg ? (uint64_t)sm_count() * per_sm : 148ull * bwd_ctas(EDGE, NO, LANES);
  if (EDGE) {  // a team's rows must all have one shift: the number of teams is a multiple of the shifts' period
    const uint64_t period = kVec<DT> / gcd64(kVec<DT>, a.x_stride % kVec<DT>), unit = period / gcd64(period, TEAMS);
    cap = cap / unit * unit;
  }
  const unsigned grid = (unsigned)(want < cap ? want : cap);
  parts = grid;
  cudaError_t e;
  if (fwd) {
    e = allow_shared(norm_fwd_kernel<DT, EDGE, NO, LANES>, ring_fwd, ready[0]);
    return e != cudaSuccess ? e : launch_overlapped(norm_fwd_kernel<DT, EDGE, NO, LANES>, dim3(grid), THREADS, ring_fwd, st, a);
  }
  if (!wg) {
    e = allow_shared(norm_bwd_kernel<DT, EDGE, NO, LANES, false>, ring_bwd, ready[1]);
    return e != cudaSuccess ? e : launch_overlapped(norm_bwd_kernel<DT, EDGE, NO, LANES, false>, dim3(grid), THREADS, ring_bwd, st, a);
  }
  e = allow_shared(norm_bwd_kernel<DT, EDGE, NO, LANES, true>, smem_wg, ready[2]);
  return e != cudaSuccess ? e : launch_overlapped(norm_bwd_kernel<DT, EDGE, NO, LANES, true>, dim3(grid), THREADS, smem_wg, st, a);
}

// The smallest team that holds the row: eight elements a lane up to 256, sixteen or twenty-four beyond.
template <int DT, bool EDGE>
cudaError_t launch_norm_shape(bool fwd, bool wg, const NormArgs& a, uint32_t elems, uint32_t& parts, cudaStream_t st) {
#define S2A_NORM(NO, LANES) \
  if (elems <= NO * LANES * 8) return launch_norm<DT, EDGE, NO, LANES>(fwd, wg, a, parts, st);
  S2A_NORM(1, 8)
  S2A_NORM(1, 16)
  S2A_NORM(1, 32)
  S2A_NORM(2, 32)
  S2A_NORM(3, 32)
  S2A_NORM(2, 64)
  S2A_NORM(3, 64)
  S2A_NORM(2, 128)
  S2A_NORM(3, 128)
  S2A_NORM(2, 256)
  S2A_NORM(3, 256)
  S2A_NORM(2, 512)
  S2A_NORM(3, 512)
  S2A_NORM(4, 512)
#undef S2A_NORM
  return cudaErrorInvalidValue;
}

template <int DT>
cudaError_t launch_norm_dt(bool fwd, bool wg, NormArgs a, uint32_t& parts, cudaStream_t st) {
  using T = typename Io<DT>::T;
  constexpr uint64_t V = kVec<DT>;
  if (a.n_rows == 1) a.x_stride = a.g_stride = a.out_stride = a.row_len;
  // how far the rows of two tensors are apart on the 16-byte grid: nowhere, if their bases and strides agree modulo it
  const auto apart = [&](const void* p, uint64_t stride) {
    return p && (((uintptr_t)p / sizeof(T) - (uintptr_t)a.x / sizeof(T)) % V != 0 || (a.n_rows > 1 && (stride - a.x_stride) % V != 0));
  };
  a.g_apart = apart(a.g, a.g_stride);
  a.out_apart = apart(a.out, a.out_stride);
  const bool shifted = ((uintptr_t)a.x / sizeof(T)) % V != 0 || (a.n_rows > 1 && a.x_stride % V != 0);
  const bool edge = shifted || a.row_len % V != 0 || a.g_apart || a.out_apart;
  const uint32_t elems = (uint32_t)(a.row_len + (shifted ? V - 1 : 0));  // with what lies before the row in its first vector
  if (elems <= 4 * 512 * 8)
    return edge ? launch_norm_shape<DT, true>(fwd, wg, a, elems, parts, st) : launch_norm_shape<DT, false>(fwd, wg, a, elems, parts, st);
  const uint64_t cap = (uint64_t)sm_count() * 4;
  const dim3 grid((unsigned)(a.n_rows < cap ? a.n_rows : cap));
  if (fwd) return launch_overlapped(norm_fwd_long_kernel<DT>, grid, kLongThreads, 0, st, a);
  if (wg) {
    const uint64_t want = (a.n_rows + 63) / 64;
    parts = (uint32_t)(want < kMaxPartials ? want : kMaxPartials);
    const cudaError_t e = launch_overlapped(norm_columns_long_kernel<DT>, dim3((a.row_len + 255) / 256, parts), 256, 0, st, a);
    if (e != cudaSuccess) return e;
  }
  return launch_overlapped(norm_bwd_long_kernel<DT>, grid, kLongThreads, 0, st, a);
}

}  // namespace

uint64_t layernorm_scratch_bytes(uint64_t n_rows, uint32_t row_len) {
  return (uint64_t)partial_cap(n_rows) * 2 * row_len * sizeof(float);
}

cudaError_t launch_layernorm_fwd(int dt, int wdt, const void* x, const void* gamma, const void* beta, void* y, float* stats,
                                 uint64_t n_rows, uint32_t row_len, uint64_t x_stride, uint64_t y_stride, float eps,
                                 cudaStream_t st) {
  NormArgs a = {};
  a.x = x;
  a.gamma = gamma;
  a.beta = beta;
  a.out = y;
  a.stats_out = stats;
  a.n_rows = n_rows;
  a.x_stride = x_stride;
  a.out_stride = y_stride;
  a.row_len = row_len;
  a.wdt = wdt;
  a.eps = eps;
  uint32_t parts = 0;
  return dt == kF32 ? launch_norm_dt<kF32>(true, false, a, parts, st) : launch_norm_dt<kBF16>(true, false, a, parts, st);
}

cudaError_t launch_layernorm_bwd(int dt, int wdt, const void* g, const void* x, const void* gamma, const float* stats,
                                 void* grad_in, void* grad_gamma, void* grad_beta, float* scratch, uint64_t n_rows,
                                 uint32_t row_len, uint64_t g_stride, uint64_t x_stride, uint64_t out_stride,
                                 cudaStream_t st) {
  const bool wg = grad_gamma || grad_beta;
  if (n_rows == 0) {  // a sum over no rows
    const size_t bytes = (size_t)row_len * (wdt == kF32 ? 4u : 2u);
    if (grad_gamma) {
      const cudaError_t e = cudaMemsetAsync(grad_gamma, 0, bytes, st);
      if (e != cudaSuccess) return e;
    }
    return grad_beta ? cudaMemsetAsync(grad_beta, 0, bytes, st) : cudaSuccess;
  }
  NormArgs a = {};
  a.x = x;
  a.g = g;
  a.gamma = gamma;
  a.out = grad_in;
  a.stats_in = stats;
  a.partials = scratch;
  a.n_rows = n_rows;
  a.x_stride = x_stride;
  a.g_stride = g_stride;
  a.out_stride = out_stride;
  a.row_len = row_len;
  a.wdt = wdt;
  uint32_t parts = 0;
  const cudaError_t e = dt == kF32 ? launch_norm_dt<kF32>(false, wg, a, parts, st) : launch_norm_dt<kBF16>(false, wg, a, parts, st);
  if (e != cudaSuccess || !wg) return e;
  return launch_overlapped(norm_reduce_kernel, dim3((row_len + 31) / 32, 2), kReduceWarps * 32, 0, st, scratch, parts, row_len,
                           grad_gamma, grad_beta, wdt);
}

}  // namespace s2a
