// Layer norm forward and backward, with the gradients of its weights.
//
//   forward   mean = sum x / L, var = sum (x - mean)^2 / L, rstd = 1 / sqrt(var + eps),
//             y = (x - mean) rstd gamma + beta; (mean, rstd) of the row are kept, 8 bytes a row
//   backward  a = g gamma, xhat = (x - mean) rstd,
//             grad_in = rstd (a - sum a / L - xhat sum(a xhat) / L),
//             grad_gamma = sum over rows of g xhat, grad_beta = sum over rows of g
//
// A row belongs to a team of TW warps and stays in its registers between the one read and the one write: NO pieces
// of eight elements a lane.  The variance is taken around the mean (two passes over registers, no difference of
// squares); warps merge (count, mean, squared deviations) with one exchange through shared memory (Chan, Golub and
// LeVeque's pairwise update).  All sums are binary32.
//
// The weights' gradients are sums over rows, so a team keeps one running sum per column in registers over all the
// rows it walks; each CTA writes one partial pair of rows to the caller's scratch and a second kernel adds the
// partials in a fixed order: no atomics, the same bits on every run.
#include "s2a_launch.h"
#include "s2a_oct.cuh"

namespace s2a {
namespace {

constexpr uint32_t kMaxRegisterRow = 16 * 32 * 32;  // 16 warps, 32 elements a lane
constexpr uint32_t kMaxPartials = 296;              // partial sums of the weights' gradients: two CTAs per SM of a B200

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
};

// Which columns a lane owns.  VEC: piece j is the eight consecutive columns from (j * LANES + lane) * 8 (whole
// 16-byte vectors).  Otherwise element i of piece j is column (j * 8 + i) * LANES + lane: neighbouring lanes on
// neighbouring elements, for rows that do not start on a 16-byte boundary.
template <bool VEC, int LANES>
__device__ __forceinline__ uint32_t column(int j, int i, uint32_t lane) {
  return VEC ? ((uint32_t)j * LANES + lane) * 8u + (uint32_t)i : (uint32_t)(j * 8 + i) * LANES + lane;
}

// A lane's share of a row as read.
template <int DT, bool VEC, int NO, int LANES>
struct Share {
  Eight<DT> p[NO];
  __device__ __forceinline__ void load(const typename Io<DT>::T* row, uint32_t lane, uint32_t L) {
#pragma unroll
    for (int j = 0; j < NO; ++j) {
      if (VEC) {
        const uint32_t c = column<VEC, LANES>(j, 0, lane);
        if (c < L) p[j].load(row + c);
        else p[j].zero();
      } else {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t c = column<VEC, LANES>(j, i, lane);
          v[i] = c < L ? Io<DT>::widen(row[c]) : 0.0f;
        }
        F2 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = f2_pack(v[2 * i], v[2 * i + 1]);
        p[j].set(w);
      }
    }
  }
};

template <int DT, bool VEC, int LANES>
__device__ __forceinline__ void store_piece(typename Io<DT>::T* row, int j, uint32_t lane, uint32_t L, const F2* v) {
  if (VEC) {
    const uint32_t c = column<VEC, LANES>(j, 0, lane);
    if (c < L) {
      Eight<DT> o;
      o.set(v);
      o.store(row + c);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t c = column<VEC, LANES>(j, i, lane);
      float lo, hi;
      f2_unpack(v[i / 2], lo, hi);
      if (c < L) row[c] = Io<DT>::narrow(i % 2 ? hi : lo);
    }
  }
}

__device__ __forceinline__ float f2_sum(F2 a) {
  float lo, hi;
  f2_unpack(a, lo, hi);
  return lo + hi;
}

// Whether both elements of pair i of piece j lie inside the row; in the vector form pieces are all in or all out.
template <bool VEC, int LANES>
__device__ __forceinline__ F2 masked(F2 v, int j, int i, uint32_t lane, uint32_t L) {
  float lo, hi;
  f2_unpack(v, lo, hi);
  return f2_pack(column<VEC, LANES>(j, 2 * i, lane) < L ? lo : 0.0f, column<VEC, LANES>(j, 2 * i + 1, lane) < L ? hi : 0.0f);
}

template <int LANES>
__device__ __forceinline__ void team_barrier(uint32_t team) {
  if (LANES > 32) asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(LANES) : "memory");
}

__host__ __device__ constexpr int threads_of(int tw) { return tw > 8 ? tw * 32 : 256; }

// ---------------------------------------------------------------- forward
template <int DT, bool VEC, int NO, int TW>
__global__ void __launch_bounds__(threads_of(TW)) norm_fwd_kernel(NormArgs a) {
  using T = typename Io<DT>::T;
  constexpr int LANES = TW * 32, TEAMS = threads_of(TW) / LANES;
  __shared__ float merge[2][TEAMS][TW][2];
  enter_grid();
  const uint32_t team = threadIdx.x / LANES, lane = threadIdx.x % LANES, warp = lane / 32, L = a.row_len;
  const float inv_l = 1.0f / (float)L;
  F2 gamma[NO][4], beta[NO][4];
  float count = 0.0f;  // elements of the row that this warp holds
#pragma unroll
  for (int j = 0; j < NO; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t c0 = column<VEC, LANES>(j, 2 * i, lane), c1 = column<VEC, LANES>(j, 2 * i + 1, lane);
      gamma[j][i] = f2_pack(a.gamma && c0 < L ? load_param(a.gamma, c0, a.wdt) : 1.0f,
                            a.gamma && c1 < L ? load_param(a.gamma, c1, a.wdt) : 1.0f);
      beta[j][i] = f2_pack(a.beta && c0 < L ? load_param(a.beta, c0, a.wdt) : 0.0f,
                           a.beta && c1 < L ? load_param(a.beta, c1, a.wdt) : 0.0f);
      count += (float)(c0 < L) + (float)(c1 < L);
    }
  count = warp_sum(count);
  const float inv_count = count > 0.0f ? 1.0f / count : 0.0f;
  const uint64_t step = (uint64_t)gridDim.x * TEAMS;
  uint32_t parity = 0;
  for (uint64_t r = (uint64_t)blockIdx.x * TEAMS + team; r < a.n_rows; r += step) {
    Share<DT, VEC, NO, LANES> raw;
    raw.load((const T*)a.x + r * a.x_stride, lane, L);
    F2 v[NO][4], sum = f2_both(0.0f);
#pragma unroll
    for (int j = 0; j < NO; ++j) {
      raw.p[j].get(v[j]);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum = f2_add(sum, v[j][i]);
    }
    float mean = warp_sum(f2_sum(sum)) * (TW == 1 ? inv_l : inv_count);
    F2 sq = f2_both(0.0f);
#pragma unroll
    for (int j = 0; j < NO; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const F2 d = masked<VEC, LANES>(f2_sub(v[j][i], f2_both(mean)), j, i, lane, L);
        sq = f2_fma(d, d, sq);
      }
    float dev = warp_sum(f2_sum(sq));
    if (TW > 1) {
      if (lane % 32 == 0) {
        merge[parity][team][warp][0] = mean * count;
        merge[parity][team][warp][1] = dev;
      }
      // the two buffers alternate: a warp writes one of them again only after the next row's barrier, which every
      // warp of the team reaches after it has read this row's values
      team_barrier<LANES>(team);
      float total = 0.0f;
#pragma unroll
      for (int w = 0; w < TW; ++w) total += merge[parity][team][w][0];
      mean = total * inv_l;
      dev = 0.0f;
#pragma unroll
      for (int w = 0; w < TW; ++w) {
        // elements of warp w, as counted above
        uint32_t n = 0;
        if (VEC) {
#pragma unroll
          for (int j = 0; j < NO; ++j) {
            const uint32_t c = ((uint32_t)j * LANES + (uint32_t)w * 32) * 8;
            n += c < L ? min(L - c, 256u) : 0u;
          }
        } else {
#pragma unroll
          for (int j = 0; j < NO * 8; ++j) {
            const uint32_t c = (uint32_t)j * LANES + (uint32_t)w * 32;
            n += c < L ? min(L - c, 32u) : 0u;
          }
        }
        const float nw = (float)n;
        const float off = n ? merge[parity][team][w][0] / nw - mean : 0.0f;
        dev += merge[parity][team][w][1] + nw * off * off;
      }
      parity ^= 1;
    }
    const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(dev * inv_l + a.eps));
    if (a.stats_out && lane == 0) ((float2*)a.stats_out)[r] = make_float2(mean, rstd);
    T* out = (T*)a.out + r * a.out_stride;
#pragma unroll
    for (int j = 0; j < NO; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[j][i] = f2_fma(f2_mul(f2_sub(v[j][i], f2_both(mean)), f2_both(rstd)), gamma[j][i], beta[j][i]);
      store_piece<DT, VEC, LANES>(out, j, lane, L, v[j]);
    }
  }
}

// ---------------------------------------------------------------- backward
template <int DT, bool VEC, int NO, int TW, bool WG>
__global__ void __launch_bounds__(threads_of(TW)) norm_bwd_kernel(NormArgs a) {
  using T = typename Io<DT>::T;
  constexpr int LANES = TW * 32, TEAMS = threads_of(TW) / LANES;
  __shared__ float2 merge[2][TEAMS][TW];
  extern __shared__ float column_sums[];  // [2][row_len], when several teams share a CTA
  enter_grid();
  const uint32_t team = threadIdx.x / LANES, lane = threadIdx.x % LANES, warp = lane / 32, L = a.row_len;
  const float inv_l = 1.0f / (float)L;
  F2 gamma[NO][4], dgamma[NO][4], dbeta[NO][4];
#pragma unroll
  for (int j = 0; j < NO; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t c0 = column<VEC, LANES>(j, 2 * i, lane), c1 = column<VEC, LANES>(j, 2 * i + 1, lane);
      gamma[j][i] = f2_pack(a.gamma && c0 < L ? load_param(a.gamma, c0, a.wdt) : 1.0f,
                            a.gamma && c1 < L ? load_param(a.gamma, c1, a.wdt) : 1.0f);
      dgamma[j][i] = dbeta[j][i] = f2_both(0.0f);
    }
  const uint64_t step = (uint64_t)gridDim.x * TEAMS;
  uint32_t parity = 0;
  for (uint64_t r = (uint64_t)blockIdx.x * TEAMS + team; r < a.n_rows; r += step) {
    Share<DT, VEC, NO, LANES> rx, rg;
    rx.load((const T*)a.x + r * a.x_stride, lane, L);
    rg.load((const T*)a.g + r * a.g_stride, lane, L);
    const float2 st = ((const float2*)a.stats_in)[r];
    const F2 mean2 = f2_both(st.x), rstd2 = f2_both(st.y);
    F2 s1 = f2_both(0.0f), s2 = f2_both(0.0f);
    // elements past the row's end have g = 0, and so no share in any sum
#pragma unroll
    for (int j = 0; j < NO; ++j) {
      F2 x[4], g[4];
      rx.p[j].get(x);
      rg.p[j].get(g);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const F2 xhat = f2_mul(f2_sub(x[i], mean2), rstd2), w = f2_mul(g[i], gamma[j][i]);
        s1 = f2_add(s1, w);
        s2 = f2_fma(w, xhat, s2);
        if (WG) {
          dgamma[j][i] = f2_fma(g[i], xhat, dgamma[j][i]);
          dbeta[j][i] = f2_add(dbeta[j][i], g[i]);
        }
      }
    }
    float c1 = warp_sum(f2_sum(s1)), c2 = warp_sum(f2_sum(s2));
    if (TW > 1) {
      if (lane % 32 == 0) merge[parity][team][warp] = make_float2(c1, c2);
      team_barrier<LANES>(team);  // alternating buffers, as in the forward kernel
      c1 = c2 = 0.0f;
#pragma unroll
      for (int w = 0; w < TW; ++w) {
        const float2 m = merge[parity][team][w];
        c1 += m.x;
        c2 += m.y;
      }
      parity ^= 1;
    }
    const F2 m1 = f2_both(c1 * inv_l), m2 = f2_both(-c2 * inv_l);
    T* out = (T*)a.out + r * a.out_stride;
#pragma unroll
    for (int j = 0; j < NO; ++j) {
      F2 x[4], g[4];
      rx.p[j].get(x);
      rg.p[j].get(g);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const F2 xhat = f2_mul(f2_sub(x[i], mean2), rstd2);
        g[i] = f2_mul(f2_fma(xhat, m2, f2_sub(f2_mul(g[i], gamma[j][i]), m1)), rstd2);
      }
      store_piece<DT, VEC, LANES>(out, j, lane, L, g);
    }
  }
  if (!WG) return;
  // The teams of a CTA add their columns one after the other, in order.
  float* part = a.partials + (uint64_t)blockIdx.x * 2 * L;
  for (uint32_t t = 0; t < TEAMS; ++t) {
    if (team == t) {
#pragma unroll
      for (int j = 0; j < NO; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t c = column<VEC, LANES>(j, i, lane);
          if (c >= L) continue;
          float dg[2], db[2];
          f2_unpack(dgamma[j][i / 2], dg[0], dg[1]);
          f2_unpack(dbeta[j][i / 2], db[0], db[1]);
          const float before_g = t ? column_sums[c] : 0.0f, before_b = t ? column_sums[L + c] : 0.0f;
          if (t + 1 < TEAMS) {
            column_sums[c] = before_g + dg[i % 2];
            column_sums[L + c] = before_b + db[i % 2];
          } else {
            part[c] = before_g + dg[i % 2];
            part[L + c] = before_b + db[i % 2];
          }
        }
    }
    if (t + 1 < TEAMS) __syncthreads();
  }
}

// Adds the partial rows: [n_part][2][row_len] -> grad_gamma, grad_beta (either may be NULL).  A CTA owns 32 columns
// of one of the two; its eight warps take every eighth partial.
__global__ void __launch_bounds__(256) norm_reduce_kernel(const float* partials, uint32_t n_part, uint32_t L, void* dgamma,
                                                          void* dbeta, int wdt) {
  __shared__ float sums[8][32];
  enter_grid();
  const uint32_t which = blockIdx.y, w = threadIdx.x / 32, c = blockIdx.x * 32 + threadIdx.x % 32;
  float acc = 0.0f;
  if (c < L)
    for (uint32_t p = w; p < n_part; p += 8) acc += partials[((uint64_t)p * 2 + which) * L + c];
  sums[w][threadIdx.x % 32] = acc;
  __syncthreads();
  void* out = which ? dbeta : dgamma;
  if (w == 0 && c < L && out) {
#pragma unroll
    for (int k = 1; k < 8; ++k) acc += sums[k][threadIdx.x];
    store_param(out, c, wdt, acc);
  }
}

// ---------------------------------------------------------------- rows too long for registers
// A CTA of 512 threads walks a row three times (sum; squared deviations; output), element by element.
constexpr int kLongThreads = 512;

__device__ __forceinline__ float cta_sum(float v, float* buf) {
  v = warp_sum(v);
  __syncthreads();
  if (threadIdx.x % 32 == 0) buf[threadIdx.x / 32] = v;
  __syncthreads();
  float t = 0.0f;
#pragma unroll
  for (int w = 0; w < kLongThreads / 32; ++w) t += buf[w];
  return t;
}

template <int DT>
__global__ void __launch_bounds__(kLongThreads) norm_fwd_long_kernel(NormArgs a) {
  using T = typename Io<DT>::T;
  __shared__ float buf[kLongThreads / 32];
  enter_grid();
  const uint32_t L = a.row_len;
  for (uint64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
    const T* x = (const T*)a.x + r * a.x_stride;
    T* y = (T*)a.out + r * a.out_stride;
    float s = 0.0f;
    for (uint32_t c = threadIdx.x; c < L; c += kLongThreads) s += Io<DT>::widen(x[c]);
    const float mean = cta_sum(s, buf) / (float)L;
    s = 0.0f;
    for (uint32_t c = threadIdx.x; c < L; c += kLongThreads) {
      const float d = Io<DT>::widen(x[c]) - mean;
      s += d * d;
    }
    const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(cta_sum(s, buf) / (float)L + a.eps));
    if (a.stats_out && threadIdx.x == 0) ((float2*)a.stats_out)[r] = make_float2(mean, rstd);
    for (uint32_t c = threadIdx.x; c < L; c += kLongThreads) {
      const float gm = a.gamma ? load_param(a.gamma, c, a.wdt) : 1.0f, bt = a.beta ? load_param(a.beta, c, a.wdt) : 0.0f;
      y[c] = Io<DT>::narrow(fmaf((Io<DT>::widen(x[c]) - mean) * rstd, gm, bt));
    }
  }
}

template <int DT>
__global__ void __launch_bounds__(kLongThreads) norm_bwd_long_kernel(NormArgs a) {
  using T = typename Io<DT>::T;
  __shared__ float buf[kLongThreads / 32];
  enter_grid();
  const uint32_t L = a.row_len;
  for (uint64_t r = blockIdx.x; r < a.n_rows; r += gridDim.x) {
    const T* x = (const T*)a.x + r * a.x_stride;
    const T* g = (const T*)a.g + r * a.g_stride;
    T* out = (T*)a.out + r * a.out_stride;
    const float2 st = ((const float2*)a.stats_in)[r];
    float s1 = 0.0f, s2 = 0.0f;
    for (uint32_t c = threadIdx.x; c < L; c += kLongThreads) {
      const float w = Io<DT>::widen(g[c]) * (a.gamma ? load_param(a.gamma, c, a.wdt) : 1.0f);
      s1 += w;
      s2 += w * ((Io<DT>::widen(x[c]) - st.x) * st.y);
    }
    const float m1 = cta_sum(s1, buf) / (float)L, m2 = cta_sum(s2, buf) / (float)L;
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
// The team that takes a row: one warp up to 1024 elements (one to four pieces of eight a lane), then twice the
// warps for each doubling (three or four pieces).
struct Team {
  int warps, pieces;
};
Team team_of(uint32_t L) {
  int tw = 1;
  while (L > (uint32_t)tw * 1024u) tw *= 2;
  return {tw, (int)((L + tw * 256 - 1) / (tw * 256))};
}

uint32_t partial_count(uint64_t n_rows, uint32_t L) {
  uint64_t want;
  if (L <= kMaxRegisterRow) {
    const int tw = team_of(L).warps;
    const uint64_t teams = threads_of(tw) / (tw * 32);
    want = (n_rows + teams - 1) / teams;
  } else {
    want = (n_rows + 63) / 64;
  }
  return (uint32_t)(want < 1 ? 1 : (want < kMaxPartials ? want : kMaxPartials));
}

template <int DT, bool VEC, int NO, int TW>
cudaError_t launch_norm(bool fwd, bool wg, const NormArgs& a, cudaStream_t st) {
  constexpr int TEAMS = threads_of(TW) / (TW * 32);
  const uint64_t want = (a.n_rows + TEAMS - 1) / TEAMS;
  if (fwd) {
    const uint64_t cap = (uint64_t)sm_count() * 4;
    return launch_overlapped(norm_fwd_kernel<DT, VEC, NO, TW>, dim3((unsigned)(want < cap ? want : cap)), threads_of(TW), 0, st, a);
  }
  if (!wg) {
    const uint64_t cap = (uint64_t)sm_count() * 4;
    return launch_overlapped(norm_bwd_kernel<DT, VEC, NO, TW, false>, dim3((unsigned)(want < cap ? want : cap)), threads_of(TW), 0, st, a);
  }
  const size_t smem = TEAMS > 1 ? (size_t)a.row_len * 8 : 0;
  return launch_overlapped(norm_bwd_kernel<DT, VEC, NO, TW, true>, dim3(partial_count(a.n_rows, a.row_len)), threads_of(TW), smem, st, a);
}

template <int DT, bool VEC>
cudaError_t launch_norm_shape(bool fwd, bool wg, const NormArgs& a, cudaStream_t st) {
  const Team t = team_of(a.row_len);
  switch (t.warps * 8 + t.pieces) {
    case 8 + 1: return launch_norm<DT, VEC, 1, 1>(fwd, wg, a, st);
    case 8 + 2: return launch_norm<DT, VEC, 2, 1>(fwd, wg, a, st);
    case 8 + 3: return launch_norm<DT, VEC, 3, 1>(fwd, wg, a, st);
    case 8 + 4: return launch_norm<DT, VEC, 4, 1>(fwd, wg, a, st);
    case 16 + 3: return launch_norm<DT, VEC, 3, 2>(fwd, wg, a, st);
    case 16 + 4: return launch_norm<DT, VEC, 4, 2>(fwd, wg, a, st);
    case 32 + 3: return launch_norm<DT, VEC, 3, 4>(fwd, wg, a, st);
    case 32 + 4: return launch_norm<DT, VEC, 4, 4>(fwd, wg, a, st);
    case 64 + 3: return launch_norm<DT, VEC, 3, 8>(fwd, wg, a, st);
    case 64 + 4: return launch_norm<DT, VEC, 4, 8>(fwd, wg, a, st);
    case 128 + 3: return launch_norm<DT, VEC, 3, 16>(fwd, wg, a, st);
    case 128 + 4: return launch_norm<DT, VEC, 4, 16>(fwd, wg, a, st);
  }
  return cudaErrorInvalidValue;
}

template <int DT>
cudaError_t launch_norm_dt(bool fwd, bool wg, const NormArgs& a, cudaStream_t st) {
  if (a.row_len > kMaxRegisterRow) {
    const uint64_t cap = (uint64_t)sm_count() * 4;
    const dim3 grid((unsigned)(a.n_rows < cap ? a.n_rows : cap));
    if (fwd) return launch_overlapped(norm_fwd_long_kernel<DT>, grid, kLongThreads, 0, st, a);
    if (wg) {
      const dim3 cols((a.row_len + 255) / 256, partial_count(a.n_rows, a.row_len));
      const cudaError_t e = launch_overlapped(norm_columns_long_kernel<DT>, cols, 256, 0, st, a);
      if (e != cudaSuccess) return e;
    }
    return launch_overlapped(norm_bwd_long_kernel<DT>, grid, kLongThreads, 0, st, a);
  }
  // whole 16-byte vectors: eight elements a piece, every row starting on a 16-byte boundary
  const uint64_t es = DT == kF32 ? 4 : 2;
  const bool vec = a.row_len % 8 == 0 && (((uintptr_t)a.x | (uintptr_t)a.out | (uintptr_t)a.g) & 15u) == 0 &&
                   ((a.n_rows == 1) || ((a.x_stride * es | a.out_stride * es | a.g_stride * es) & 15u) == 0);
  return vec ? launch_norm_shape<DT, true>(fwd, wg, a, st) : launch_norm_shape<DT, false>(fwd, wg, a, st);
}

}  // namespace

uint64_t layernorm_scratch_bytes(uint64_t n_rows, uint32_t row_len) {
  return (uint64_t)partial_count(n_rows, row_len) * 2 * row_len * sizeof(float);
}

cudaError_t launch_layernorm_fwd(int dt, int wdt, const void* x, const void* gamma, const void* beta, void* y, float* stats,
                                 uint64_t n_rows, uint32_t row_len, uint64_t x_stride, uint64_t y_stride, float eps,
                                 cudaStream_t st) {
  NormArgs a{x, nullptr, gamma, beta, y, nullptr, stats, nullptr, n_rows, x_stride, 0, y_stride, row_len, wdt, eps};
  return dt == kF32 ? launch_norm_dt<kF32>(true, false, a, st) : launch_norm_dt<kBF16>(true, false, a, st);
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
  NormArgs a{x, g, gamma, nullptr, grad_in, stats, nullptr, scratch, n_rows, x_stride, g_stride, out_stride, row_len, wdt, 0.0f};
  const cudaError_t e = dt == kF32 ? launch_norm_dt<kF32>(false, wg, a, st) : launch_norm_dt<kBF16>(false, wg, a, st);
  if (e != cudaSuccess || !wg) return e;
  return launch_overlapped(norm_reduce_kernel, dim3((row_len + 31) / 32, 2), 256, 0, st, scratch,
                           partial_count(n_rows, row_len), row_len, grad_gamma, grad_beta, wdt);
}

}  // namespace s2a
