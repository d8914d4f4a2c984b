// Host side of rotary positions and of the norms of queries and keys, the table of turns, and the sum of the weights' partial
// gradients; the kernels are in s2a_rope.cuh.
#include <math.h>

#include <algorithm>

#include "s2a_launch.h"
#include "s2a_oct.cuh"

namespace s2a {

// s2a_rope.cuh: rows of 32, 64, 96, 128, 160, 192 or 256 elements that turn as a whole, on the 16-byte grid; and any others (MULTI: tokens with fewer rows than
// a group has)
template <int DT>
cudaError_t launch_rope_whole(int mode, const RopeArgs& a, unsigned grid, cudaStream_t st);
template <int DT, bool MULTI>
cudaError_t launch_rope_any(int mode, uint32_t V, uint32_t W, const RopeArgs& a, unsigned grid, cudaStream_t st);

namespace {

constexpr int kWarps = 8;         // as in the kernels
constexpr int kLaneElems = 16;

// grad_gamma of queries (blockIdx.y = 0) and keys: the CTAs' partial rows added in a fixed order and in 64 bits, a column a lane, a warp's share of
// the rows in flight at once.
constexpr int kReduceWarps = 16;
constexpr int kReduceRows = (kMaxRopePartials + kReduceWarps - 1) / kReduceWarps;  // of a warp

__global__ void __launch_bounds__(kReduceWarps * 32) qknorm_reduce_kernel(const float* partials, uint32_t ctas0, uint32_t ctas, uint32_t D,
                                                                         void* gq, void* gk, int wdt) {
  __shared__ double buf[kReduceWarps][33];
  enter_grid();
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, d = blockIdx.x * 32 + lane;
  const uint32_t from = blockIdx.y ? ctas0 : 0, to = blockIdx.y ? ctas : ctas0;
  void* out = blockIdx.y ? gk : gq;
  float p[kReduceRows];
#pragma unroll
  for (int i = 0; i < kReduceRows; ++i) {
    const uint32_t r = from + warp + i * kReduceWarps;
    p[i] = d < D && r < to ? partials[(uint64_t)r * D + d] : 0.0f;
  }
  double s = 0.0, t = 0.0;  // an addition waits for the one before it
#pragma unroll
  for (int i = 0; i < kReduceRows; ++i) (i % 2 ? t : s) += (double)p[i];
  buf[warp][lane] = s + t;
  __syncthreads();
  if (warp == 0 && d < D && out) {
    s = 0.0;
#pragma unroll
    for (int w = 0; w < kReduceWarps; ++w) s += buf[w][lane];
    store_param(out, d, wdt, (float)s);
  }
}

// Whether a tensor of heads may be read in vectors of `bytes`.
bool fits(const HeadsArg& h, uint32_t heads, uint32_t es, uint32_t bytes) {
  if (heads == 0 || !h.data) return true;
  return (uintptr_t)h.data % bytes == 0 && (h.batch * es) % bytes == 0 && (h.token * es) % bytes == 0 && (h.head * es) % bytes == 0;
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
  // W: the widest vector that divides a row and every address.  V: the widest within it that divides what turns and what does not: in the
  // layout of halves the half that turns and the rest, interleaved (where pairs lie within vectors) all that turns.
  const uint32_t widest = 16 / es;
  uint32_t W = widest;
  for (; W > 1; W /= 2) {
    bool ok = a.head_dim % W == 0;
    for (int i = 0; i < 2 && ok; ++i)
      ok = fits(a.in[i], a.heads[i], es, W * es) && fits(a.grad[i], a.heads[i], es, W * es) && fits(a.out[i], a.heads[i], es, W * es);
    if (ok) break;
  }
  uint32_t V = W;
  while (V > 1 && (a.interleaved ? (2 * a.pairs) % V : a.pairs % V || (a.head_dim - 2 * a.pairs) % V)) V /= 2;
  if (W != widest) W = V = V > 2 ? 2 : V;
  const uint32_t K = kLaneElems / (2 * V);
  const bool inside = a.interleaved && V > 1;  // pairs within vectors
  a.turn_slots = a.pairs / V;
  a.slots = inside ? (a.head_dim / V + 1) / 2 : a.turn_slots + (a.head_dim - 2 * a.pairs + 2 * V - 1) / (2 * V);
  a.lanes = (a.slots + K - 1) / K;
  a.rows_per_warp = 32 / a.lanes;
  a.inv_dim = 1.0f / (float)a.head_dim;
  a.pairs_inverse = a.pairs ? (1048576u + a.pairs - 1) / a.pairs : 0u;
  // A group is rows of one token; or, where those are at most half of what a group takes, the rows of several tokens.  Where
  // the norms' backward has many query heads, few key heads alone do not call for it: groups of several tokens walk the sequences
  // for every row, and [1, 8654, 32 + 1, 64] takes 68 us with them and 32 us without, [1, 4298, 8 + 1, 96] 30 and 17 us (binary32).
  const auto few = [&](uint32_t rows) { return rows != 0 && 2 * rows <= a.rows_per_warp; };
  const bool multi = mode == kRopeBwdNorm ? few(a.heads[0]) && (a.heads[1] == 0 || few(a.heads[1])) : few(heads);
  // A warp each for the groups, until the GPU is full; then shares.  `which`: the forward kernels (and queries), keys.
  uint64_t items[2] = {0, 0};
  const auto group = [&](uint32_t rows, int which) {
    a.group_tokens[which] = multi && few(rows) ? a.rows_per_warp / rows : 1;
    a.step_b[which] = a.group_tokens[which] % a.batch;
    a.step_t[which] = a.group_tokens[which] / a.batch;
    items[which] = a.group_tokens[which] > 1 ? (tokens + a.group_tokens[which] - 1) / a.group_tokens[which]
                                             : tokens * ((rows + a.rows_per_warp - 1) / a.rows_per_warp);
  };
  const auto cut = [&](uint32_t ctas, int which) {
    const uint64_t warps = (uint64_t)ctas * kWarps;
    a.share[which] = (uint32_t)(items[which] / warps);
    a.more[which] = (uint32_t)(items[which] % warps);
  };
  const auto ctas_for = [&](uint64_t n, uint64_t cap) { return (uint32_t)std::min<uint64_t>((n + kWarps - 1) / kWarps, cap); };
  unsigned grid;
  if (mode == kRopeBwdNorm) {
    group(a.heads[0], 0);
    group(a.heads[1], 1);
    const uint64_t cap = kMaxRopePartials, share0 = cap * items[0] / (items[0] + items[1]);
    a.ctas0 = items[0] ? ctas_for(items[0], items[1] ? std::min(std::max<uint64_t>(share0, 1), cap - 1) : cap) : 0;
    const uint32_t ctas1 = items[1] ? ctas_for(items[1], cap - a.ctas0) : 0;
    grid = a.ctas0 + ctas1;
    if (items[0]) cut(a.ctas0, 0);
    if (items[1]) cut(ctas1, 1);
    a.partials = sums ? scratch : nullptr;
  } else {
    group(heads, 0);
    grid = ctas_for(items[0], (uint64_t)sm_count() * (multi ? 2 : 3));
    cut(grid, 0);
  }
  if ((items[0] | items[1]) >> 32) return cudaErrorInvalidValue;  // more rows than any memory holds
  // from here on strides are in bytes
  for (HeadsArg* h : {&a.in[0], &a.in[1], &a.grad[0], &a.grad[1], &a.out[0], &a.out[1]}) {
    h->batch *= es;
    h->token *= es;
    h->head *= es;
  }
  const bool whole = !multi && V == widest && 2 * a.pairs == a.head_dim && a.head_dim % 32 == 0 && a.head_dim <= 256 && a.head_dim != 224;
  const cudaError_t e = whole ? (dt == kF32 ? launch_rope_whole<kF32>(mode, a, grid, st) : launch_rope_whole<kBF16>(mode, a, grid, st))
                        : multi ? (dt == kF32 ? launch_rope_any<kF32, true>(mode, V, W, a, grid, st) : launch_rope_any<kBF16, true>(mode, V, W, a, grid, st))
                                : (dt == kF32 ? launch_rope_any<kF32, false>(mode, V, W, a, grid, st) : launch_rope_any<kBF16, false>(mode, V, W, a, grid, st));
  if (e != cudaSuccess || !sums) return e;
  return launch_overlapped(qknorm_reduce_kernel, dim3((a.head_dim + 31) / 32, 2), kReduceWarps * 32, 0, st, scratch, a.ctas0, grid, a.head_dim,
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
