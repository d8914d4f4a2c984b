// Rotary positions, and the norms of queries and keys with the rotation in the same pass, forward and backward.
//
// A head's row of D elements turns in pairs: (a, b) -> (a cos - b sin, a sin + b cos), pair i of a token at position p by the
// angle p * w_i; backward turns by the opposite angle.  The phase is exact at any position: the table holds w_i / (2 pi) as a
// 64-bit binary fraction of a turn, so that turn * p modulo 2^64 is the angle's fraction of a turn (the error of the
// table's last bit times p: below 2^-33 of a turn for |p| < 2^31).  One integer product takes the place of a table of cosines over all positions
// or of products in 64 bits.
//
// With the norm: y = R(x * rstd * gamma), rstd = 1 / sqrt(mean(x^2) + eps).  Backward keeps nothing but x: with u = R^-1(g),
// a = u * gamma, xhat = x * rstd:  grad_x = rstd * (a - xhat * mean(a * xhat)),  grad_gamma = sum of u * xhat; the row is in
// registers anyway, so rstd costs one more sum and no memory.
//
// All of it is bound by memory: each row is read once (backward: g and x) and written once.  A lane owns 16 elements of a row
// as K slots of two vectors of V; a slot holds V pairs, or 2 V of the elements that do not turn.  The two vectors of a turning
// slot are rot / 2 elements apart in both layouts, so that pairs never cross lanes and a warp's accesses are alike.  A warp
// takes 32 / L rows (L lanes a row) of one token at a time, all heads of queries and keys in turn, so that a token's
// cosines and sines are computed once, one or a few a lane, and shared through the warp's own shared memory.
#include "s2a_launch.h"
#include "s2a_oct.cuh"

namespace s2a {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kLaneElems = 16;
constexpr int kMaxPairs = kMaxHeadDim / 2;

// Where a warp's lanes stand in the rows they take together.
struct Lane {
  uint32_t slot, row;  // slot of k = 0 in the row, row of the group
  bool on;
};

__device__ __forceinline__ float2 phase(uint64_t turn, int64_t pos, float scale, bool back) {
  // The fraction's top 32 bits: a quarter turn to the nearest, and what is left of it, at most an eighth of a turn, which a
  // float holds to 2^-28 of a turn
  const uint32_t top = (uint32_t)((turn * (uint64_t)pos) >> 32);
  const uint32_t quarter = (top + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(top - (quarter << 30)) * 4.656612873077393e-10f;  // in half turns: 2^-31
  float s, c;
  sincospif(x, &s, &c);
  if (quarter & 1u) {
    const float t = c;
    c = -s;
    s = t;
  }
  if (quarter & 2u) {
    c = -c;
    s = -s;
  }
  return make_float2(c * scale, (back ? -s : s) * scale);
}

// The warp's cosines and sines of one token.
__device__ __forceinline__ void warp_phases(const RopeArgs& a, uint32_t b, uint32_t t, float* cs, float* sn) {
  const uint32_t lane = threadIdx.x & 31u;
  for (uint32_t i = lane; i < a.pairs; i += 32) {
    const ulonglong2 e = __ldg((const ulonglong2*)a.table + i);
    int64_t pos = a.first + t;
    if (a.positions) {
      const uint64_t axis = e.y < a.axes ? e.y : a.axes - 1;
      pos = __ldg(a.positions + axis * a.pos_axis + b * a.pos_batch + t);
    }
    const float2 v = phase(e.x, pos, a.scale, a.back);
    cs[i] = v.x;
    sn[i] = v.y;
  }
  __syncwarp();
}

template <int BYTES> struct RawOf;
template <> struct RawOf<16> { using T = uint4; };
template <> struct RawOf<8> { using T = uint2; };
template <> struct RawOf<4> { using T = uint32_t; };
template <> struct RawOf<2> { using T = uint16_t; };

template <int DT, int V>
struct Slot {
  using Raw = typename RawOf<V * Io<DT>::kBytes>::T;
  union {
    Raw r;
    uint32_t w[(V * Io<DT>::kBytes + 3) / 4];
  };
  __device__ __forceinline__ Slot() {}
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < (V * Io<DT>::kBytes + 3) / 4; ++i) w[i] = 0u;
  }
  __device__ __forceinline__ void load(const typename Io<DT>::T* p) { r = *(const Raw*)p; }
  __device__ __forceinline__ void store(typename Io<DT>::T* p) const { *(Raw*)p = r; }
  __device__ __forceinline__ void get(float* f) const {
    if constexpr (DT == kF32) {
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = __uint_as_float(w[i]);
    } else if constexpr (V == 1) {
      f[0] = __uint_as_float((uint32_t)r << 16);
    } else {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ void set(const float* f) {
    if constexpr (DT == kF32) {
#pragma unroll
      for (int i = 0; i < V; ++i) w[i] = __float_as_uint(f[i]);
    } else if constexpr (V == 1) {
      r = __bfloat16_as_ushort(__float2bfloat16_rn(f[0]));
    } else {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) w[i] = f2_to_bf16x2(f2_pack(f[2 * i], f[2 * i + 1]));
    }
  }
};

// A lane's places in a row, the same in every row of a launch: the two vectors of each slot, and which of them exist.
template <int V, int K, bool INTER>
struct Places {
  uint32_t at[K], to[K];  // elements of the first and the second vector
  uint32_t first, second;  // bits: which of them exist
  uint32_t pair[K], pair2[K];  // first pair of the first and, interleaved, of the second vector
  uint32_t turns;          // bits: slots that turn
  __device__ __forceinline__ Places(const RopeArgs& a, const Lane& l) {
    first = second = turns = 0u;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t s = l.slot + k * a.lanes;
      at[k] = to[k] = pair[k] = pair2[k] = 0u;
      if (!l.on || s >= a.slots) continue;
      first |= 1u << k;
      if (s < a.turn_slots) {
        turns |= 1u << k;
        second |= 1u << k;
        if (V == 1) {  // single pairs: adjacent, or half apart
          at[k] = a.interleaved ? 2 * s : s;
          to[k] = a.interleaved ? 2 * s + 1 : s + a.pairs;
          pair[k] = s;
        } else {
          at[k] = V * s;
          to[k] = V * s + a.pairs;
          pair[k] = INTER ? at[k] / 2 : at[k];
          pair2[k] = INTER ? to[k] / 2 : 0u;
        }
      } else {
        at[k] = 2 * a.pairs + 2 * V * (s - a.turn_slots);
        to[k] = at[k] + V;
        if (to[k] < a.head_dim) second |= 1u << k;
        else to[k] = at[k];
      }
    }
  }
};

// A lane's cosines and sines; a slot that does not turn has 1 and 0.
template <int V, int K, bool INTER>
struct Angles {
  float c[K][V], s[K][V];
  __device__ __forceinline__ void read(const Places<V, K, INTER>& p, const float* cs, const float* sn) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const bool turns = (p.turns >> k) & 1u;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const uint32_t i = !INTER ? p.pair[k] + j : (j < V / 2 ? p.pair[k] + j : p.pair2[k] + j - V / 2);
        c[k][j] = turns ? cs[i] : 1.0f;
        s[k][j] = turns ? sn[i] : 0.0f;
      }
    }
  }
  __device__ __forceinline__ void turn(int k, float* a, float* b) const {
    if constexpr (!INTER) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float u = a[j] * c[k][j] - b[j] * s[k][j];
        b[j] = a[j] * s[k][j] + b[j] * c[k][j];
        a[j] = u;
      }
    } else {
#pragma unroll
      for (int j = 0; j < V / 2; ++j) {
        float u = a[2 * j] * c[k][j] - a[2 * j + 1] * s[k][j];
        a[2 * j + 1] = a[2 * j] * s[k][j] + a[2 * j + 1] * c[k][j];
        a[2 * j] = u;
        u = b[2 * j] * c[k][V / 2 + j] - b[2 * j + 1] * s[k][V / 2 + j];
        b[2 * j + 1] = b[2 * j] * s[k][V / 2 + j] + b[2 * j + 1] * c[k][V / 2 + j];
        b[2 * j] = u;
      }
    }
  }
};

template <int DT, int V, int K>
struct Row {
  Slot<DT, V> a[K], b[K];
  template <typename P>
  __device__ __forceinline__ void load(const typename Io<DT>::T* row, const P& p, bool on) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (on && ((p.first >> k) & 1u)) a[k].load(row + p.at[k]);
      else a[k].zero();
      if (on && ((p.second >> k) & 1u)) b[k].load(row + p.to[k]);
      else b[k].zero();
    }
  }
  template <typename P>
  __device__ __forceinline__ void store(typename Io<DT>::T* row, const P& p, bool on) const {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (on && ((p.first >> k) & 1u)) a[k].store(row + p.at[k]);
      if (on && ((p.second >> k) & 1u)) b[k].store(row + p.to[k]);
    }
  }
};

// Sum over the `lanes` neighbouring lanes of a row, at every one of them.  The lanes of a row are any number up to 32.
__device__ __forceinline__ float row_sum(float v, uint32_t in_row, uint32_t lanes) {
  for (uint32_t o = 1; o < lanes; o <<= 1) {
    const float w = __shfl_down_sync(0xffffffffu, v, o);
    if (in_row + o < lanes) v += w;
  }
  return __shfl_sync(0xffffffffu, v, (threadIdx.x & 31u) - in_row);
}

template <int V, int K, typename P>
__device__ __forceinline__ void load_gamma(const void* gamma, int wdt, const P& p, float (&ga)[K][V], float (&gb)[K][V]) {
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      ga[k][j] = gamma && ((p.first >> k) & 1u) ? load_param(gamma, p.at[k] + j, wdt) : 1.0f;
      gb[k][j] = gamma && ((p.second >> k) & 1u) ? load_param(gamma, p.to[k] + j, wdt) : 1.0f;
    }
}

enum { kPlain = 0, kNorm = 1 };

// Forward of both operators, and the rotation's backward.  A unit is a token, or one of `parts` parts of its groups of rows:
// the groups of the queries' heads come first, then those of the keys'.
template <int DT, int V, bool INTER, int NORM>
__global__ void __launch_bounds__(kThreads) rope_kernel(RopeArgs a) {
  using T = typename Io<DT>::T;
  constexpr int K = kLaneElems / (2 * V);
  __shared__ __align__(16) float cs_all[kWarps][kMaxPairs], sn_all[kWarps][kMaxPairs];
  enter_grid();
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  Lane l;
  l.row = lane / a.lanes;
  l.slot = lane - l.row * a.lanes;
  l.on = l.row < a.rows_per_warp;
  const Places<V, K, INTER> p(a, l);
  const uint32_t groups0 = (a.heads[0] + a.rows_per_warp - 1) / a.rows_per_warp;
  const uint32_t groups = groups0 + (a.heads[1] + a.rows_per_warp - 1) / a.rows_per_warp;
  float* cs = cs_all[warp];
  float* sn = sn_all[warp];
  for (uint64_t unit = (uint64_t)blockIdx.x * kWarps + warp; unit < a.units; unit += (uint64_t)gridDim.x * kWarps) {
    const uint32_t n = (uint32_t)(unit / a.parts), part = (uint32_t)(unit % a.parts);
    const uint32_t b = n / a.tokens, t = n - b * a.tokens;
    const T* in[2];
    T* out[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      in[i] = (const T*)a.in[i].data + b * a.in[i].batch + t * a.in[i].token;
      out[i] = (T*)a.out[i].data + b * a.out[i].batch + t * a.out[i].token;
    }
    Angles<V, K, INTER> angles;
    __syncwarp();  // the last unit's cosines have been read
    warp_phases(a, b, t, cs, sn);
    angles.read(p, cs, sn);
    float ga[K][V], gb[K][V];
    int kind = -1;
    for (uint32_t i = part; i < groups; i += a.parts) {
      const int which = i >= groups0;
      const uint32_t h = (which ? i - groups0 : i) * a.rows_per_warp + l.row;
      const bool on = l.on && h < a.heads[which];
      Row<DT, V, K> x;
      x.load(in[which] + (on ? h * a.in[which].head : 0), p, on);
      if (NORM == kNorm && which != kind) {
        load_gamma<V, K>(a.gamma[which], a.wdt, p, ga, gb);
        kind = which;
      }
      float fa[K][V], fb[K][V];
#pragma unroll
      for (int k = 0; k < K; ++k) {
        x.a[k].get(fa[k]);
        x.b[k].get(fb[k]);
      }
      if (NORM == kNorm) {
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
          for (int j = 0; j < V; ++j) sum = fmaf(fa[k][j], fa[k][j], fmaf(fb[k][j], fb[k][j], sum));
        const float rstd = __frsqrt_rn(row_sum(sum, l.slot, a.lanes) * a.inv_dim + a.eps);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
          for (int j = 0; j < V; ++j) {
            fa[k][j] = fa[k][j] * rstd * ga[k][j];
            fb[k][j] = fb[k][j] * rstd * gb[k][j];
          }
      }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        angles.turn(k, fa[k], fb[k]);
        x.a[k].set(fa[k]);
        x.b[k].set(fb[k]);
      }
      x.store(out[which] + (on ? h * a.out[which].head : 0), p, on);
    }
  }
}

// The norm's backward.  A CTA takes rows of queries or of keys only (the first ctas0 CTAs those of queries), so that a lane
// keeps one set of sums for grad_gamma; they are added up over the CTA's rows and left in the scratch, one row of head_dim a CTA.
template <int DT, int V, bool INTER>
__global__ void __launch_bounds__(kThreads) qknorm_bwd_kernel(RopeArgs a) {
  using T = typename Io<DT>::T;
  constexpr int K = kLaneElems / (2 * V);
  __shared__ __align__(16) float shared[kWarps * 32 * kLaneElems];
  static_assert(2 * kMaxPairs * kWarps <= kWarps * 32 * kLaneElems, "the phases fit in the sums' place");
  enter_grid();
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  Lane l;
  l.row = lane / a.lanes;
  l.slot = lane - l.row * a.lanes;
  l.on = l.row < a.rows_per_warp;
  const Places<V, K, INTER> p(a, l);
  const int which = blockIdx.x >= a.ctas0;
  const uint32_t cta = which ? blockIdx.x - a.ctas0 : blockIdx.x, ctas = which ? gridDim.x - a.ctas0 : a.ctas0;
  const uint32_t heads = a.heads[which], groups = (heads + a.rows_per_warp - 1) / a.rows_per_warp;
  const uint32_t parts = a.parts < groups ? a.parts : groups;
  const uint64_t units = (uint64_t)a.batch * a.tokens * parts;
  float* cs = shared + warp * 2 * kMaxPairs;
  float* sn = cs + kMaxPairs;
  float ga[K][V], gb[K][V], sa[K][V], sb[K][V];
  load_gamma<V, K>(a.gamma[which], a.wdt, p, ga, gb);
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j) sa[k][j] = sb[k][j] = 0.0f;
  for (uint64_t unit = (uint64_t)cta * kWarps + warp; unit < units; unit += (uint64_t)ctas * kWarps) {
    const uint32_t n = (uint32_t)(unit / parts), part = (uint32_t)(unit % parts);
    const uint32_t b = n / a.tokens, t = n - b * a.tokens;
    const T* x0 = (const T*)a.in[which].data + b * a.in[which].batch + t * a.in[which].token;
    const T* g0 = (const T*)a.grad[which].data + b * a.grad[which].batch + t * a.grad[which].token;
    T* out = (T*)a.out[which].data + b * a.out[which].batch + t * a.out[which].token;
    Angles<V, K, INTER> angles;
    __syncwarp();
    warp_phases(a, b, t, cs, sn);
    angles.read(p, cs, sn);
    for (uint32_t i = part; i < groups; i += parts) {
      const uint32_t h = i * a.rows_per_warp + l.row;
      const bool on = l.on && h < heads;
      Row<DT, V, K> x, g;
      x.load(x0 + (on ? h * a.in[which].head : 0), p, on);
      g.load(g0 + (on ? h * a.grad[which].head : 0), p, on);
      float xa[K][V], xb[K][V], ua[K][V], ub[K][V];
      float sum = 0.0f, along = 0.0f;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        x.a[k].get(xa[k]);
        x.b[k].get(xb[k]);
        g.a[k].get(ua[k]);
        g.b[k].get(ub[k]);
        angles.turn(k, ua[k], ub[k]);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          sum = fmaf(xa[k][j], xa[k][j], fmaf(xb[k][j], xb[k][j], sum));
          along = fmaf(ua[k][j] * ga[k][j], xa[k][j], fmaf(ub[k][j] * gb[k][j], xb[k][j], along));
        }
      }
      const float rstd = __frsqrt_rn(row_sum(sum, l.slot, a.lanes) * a.inv_dim + a.eps);
      const float mean = row_sum(along, l.slot, a.lanes) * rstd * a.inv_dim;  // of a * xhat
      if (on) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float ha = xa[k][j] * rstd, hb = xb[k][j] * rstd;
            sa[k][j] = fmaf(ua[k][j], ha, sa[k][j]);
            sb[k][j] = fmaf(ub[k][j], hb, sb[k][j]);
            ua[k][j] = (ua[k][j] * ga[k][j] - ha * mean) * rstd;
            ub[k][j] = (ub[k][j] * gb[k][j] - hb * mean) * rstd;
          }
          x.a[k].set(ua[k]);
          x.b[k].set(ub[k]);
        }
        x.store(out + h * a.out[which].head, p, true);
      }
    }
  }
  if (!a.partials) return;
  __syncthreads();  // the phases' place becomes the sums'
  const uint32_t D = a.head_dim, rows = kWarps * a.rows_per_warp;
  float* mine = shared + (warp * a.rows_per_warp + l.row) * D;
  if (l.on) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if ((p.first >> k) & 1u) mine[p.at[k] + j] = sa[k][j];
        if ((p.second >> k) & 1u) mine[p.to[k] + j] = sb[k][j];
      }
  }
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < D; d += kThreads) {
    float s = 0.0f;
    for (uint32_t r = 0; r < rows; ++r) s += shared[r * D + d];
    a.partials[(uint64_t)blockIdx.x * D + d] = s;
  }
}

// grad_gamma of queries (blockIdx.y = 0) and keys: the CTAs' partial rows added in a fixed order, a column a lane.
__global__ void __launch_bounds__(1024) qknorm_reduce_kernel(const float* partials, uint32_t ctas0, uint32_t ctas, uint32_t D,
                                                             void* gq, void* gk, int wdt) {
  __shared__ float buf[32][33];
  enter_grid();
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, d = blockIdx.x * 32 + lane;
  const uint32_t from = blockIdx.y ? ctas0 : 0, to = blockIdx.y ? ctas : ctas0;
  void* out = blockIdx.y ? gk : gq;
  float s = 0.0f;
  if (d < D)
    for (uint32_t r = from + warp; r < to; r += 32) s += partials[(uint64_t)r * D + d];
  buf[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && d < D && out) {
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < 32; ++w) s += buf[w][lane];
    store_param(out, d, wdt, s);
  }
}

// ---------------------------------------------------------------- host side
// Whether a tensor of heads may be read in vectors of `bytes`.
bool fits(const HeadsArg& h, uint32_t heads, uint32_t es, uint32_t bytes) {
  if (heads == 0 || !h.data) return true;
  return (uintptr_t)h.data % bytes == 0 && (h.batch * es) % bytes == 0 && (h.token * es) % bytes == 0 && (h.head * es) % bytes == 0;
}

template <int DT, int V, bool INTER>
cudaError_t launch_one(int mode, const RopeArgs& a, unsigned grid, cudaStream_t st) {
  if (mode == kRopeBwdNorm) return launch_overlapped(qknorm_bwd_kernel<DT, V, INTER>, dim3(grid), kThreads, 0, st, a);
  if (mode == kRopeFwdNorm) return launch_overlapped(rope_kernel<DT, V, INTER, kNorm>, dim3(grid), kThreads, 0, st, a);
  return launch_overlapped(rope_kernel<DT, V, INTER, kPlain>, dim3(grid), kThreads, 0, st, a);
}

template <int DT, int V>
cudaError_t launch_layout(int mode, const RopeArgs& a, unsigned grid, cudaStream_t st) {
  if constexpr (V > 1)
    if (a.interleaved) return launch_one<DT, V, true>(mode, a, grid, st);
  return launch_one<DT, V, false>(mode, a, grid, st);
}

}  // namespace

uint64_t qknorm_scratch_bytes(uint32_t head_dim) { return (uint64_t)kMaxRopePartials * head_dim * sizeof(float); }

cudaError_t launch_rope(int mode, int dt, RopeArgs a, void* grad_gamma_q, void* grad_gamma_k, float* scratch, cudaStream_t st) {
  const uint64_t tokens = (uint64_t)a.batch * a.tokens;
  const uint32_t heads = a.heads[0] + a.heads[1];
  const bool sums = mode == kRopeBwdNorm && (grad_gamma_q || grad_gamma_k);
  if (tokens == 0 || heads == 0) {  // sums over no rows
    const size_t bytes = (size_t)a.head_dim * (a.wdt == kF32 ? 4u : 2u);
    if (sums && grad_gamma_q) {
      const cudaError_t e = cudaMemsetAsync(grad_gamma_q, 0, bytes, st);
      if (e != cudaSuccess) return e;
    }
    return sums && grad_gamma_k ? cudaMemsetAsync(grad_gamma_k, 0, bytes, st) : cudaSuccess;
  }
  const uint32_t es = dt == kF32 ? 4u : 2u;
  // the widest vector that divides the turning half, the rest of the row, and every address
  uint32_t V = 16 / es;
  for (; V > 1; V /= 2) {
    bool ok = a.pairs % V == 0 && (a.head_dim - 2 * a.pairs) % V == 0;
    for (int i = 0; i < 2 && ok; ++i)
      ok = fits(a.in[i], a.heads[i], es, V * es) && fits(a.grad[i], a.heads[i], es, V * es) && fits(a.out[i], a.heads[i], es, V * es);
    if (ok) break;
  }
  const uint32_t K = kLaneElems / (2 * V);
  a.turn_slots = a.pairs / V;
  a.slots = a.turn_slots + (a.head_dim - 2 * a.pairs + 2 * V - 1) / (2 * V);
  a.lanes = (a.slots + K - 1) / K;
  a.rows_per_warp = 32 / a.lanes;
  a.inv_dim = 1.0f / (float)a.head_dim;
  const uint32_t sms = (uint32_t)sm_count();
  const uint32_t groups0 = (a.heads[0] + a.rows_per_warp - 1) / a.rows_per_warp;
  const uint32_t groups = groups0 + (a.heads[1] + a.rows_per_warp - 1) / a.rows_per_warp;
  // few tokens: a token's groups are shared by several warps, until every SM has its warps
  const uint64_t want = (uint64_t)sms * kWarps * 4;
  const uint64_t shares = (want + tokens - 1) / tokens;
  a.parts = (uint32_t)(shares < groups ? shares : groups);
  a.units = tokens * a.parts;
  unsigned grid;
  if (mode == kRopeBwdNorm) {
    const uint64_t need = (a.units + kWarps - 1) / kWarps;
    uint32_t cap = 148 * 2;
    if (need < cap) cap = (uint32_t)need;
    a.ctas0 = a.heads[1] == 0 ? cap : (a.heads[0] == 0 ? 0 : (uint32_t)((uint64_t)cap * a.heads[0] / heads));
    if (a.heads[0] && a.ctas0 == 0) a.ctas0 = 1;
    grid = cap;
    if (a.heads[1] && a.ctas0 >= cap) grid = a.ctas0 + 1;
    a.partials = sums ? scratch : nullptr;
  } else {
    const uint64_t need = (a.units + kWarps - 1) / kWarps, cap = (uint64_t)sms * 16;
    grid = (unsigned)(need < cap ? need : cap);
  }
  cudaError_t e;
  if (dt == kF32)
    e = V == 4 ? launch_layout<kF32, 4>(mode, a, grid, st) : (V == 2 ? launch_layout<kF32, 2>(mode, a, grid, st) : launch_layout<kF32, 1>(mode, a, grid, st));
  else
    e = V == 8 ? launch_layout<kBF16, 8>(mode, a, grid, st)
               : (V == 4 ? launch_layout<kBF16, 4>(mode, a, grid, st)
                         : (V == 2 ? launch_layout<kBF16, 2>(mode, a, grid, st) : launch_layout<kBF16, 1>(mode, a, grid, st)));
  if (e != cudaSuccess || !sums) return e;
  return launch_overlapped(qknorm_reduce_kernel, dim3((a.head_dim + 31) / 32, 2), 1024, 0, st, scratch, a.ctas0, grid, a.head_dim,
                           grad_gamma_q, grad_gamma_k, a.wdt);
}

// ---------------------------------------------------------------- the table of turns
void rope_table(uint64_t* out, uint32_t pairs, double base, int scaling, double factor, double original, double slow, double fast,
                uint32_t axes) {
  const uint32_t each = pairs / axes;
  const long double tau = 6.283185307179586476925286766559005768L;
  long double b = base;
  if (scaling == kRopeScaleBase && each > 1) b *= powl((long double)factor, (long double)each / (each - 1));
  for (uint32_t i = 0; i < pairs; ++i) {
    const uint32_t j = i % each;
    long double turn = powl(b, -(long double)j / each) / tau;
    if (scaling == kRopeScaleLinear) turn /= factor;
    if (scaling == kRopeScaleParts) {
      long double keep = (original * turn - slow) / (fast - slow);
      keep = keep < 0.0L ? 0.0L : (keep > 1.0L ? 1.0L : keep);
      turn *= keep + (1.0L - keep) / factor;
    }
    turn -= floorl(turn);  // whole turns change nothing
    out[2 * i] = (uint64_t)nearbyintl(ldexpl(turn, 63)) << 1;
    out[2 * i + 1] = i / each;
  }
}

}  // namespace s2a
