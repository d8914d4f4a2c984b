// Host side of rotary positions and of the norms of queries and keys, the table of turns, and the sum of the weights' partial
// gradients; the kernels are in s2a_rope.cuh.
#include <math.h>

#include <algorithm>

#include "s2a_launch.h"
#include "s2a_oct.cuh"

namespace s2a {

template <int DT>
cudaError_t launch_rope_kernel(int mode, uint32_t V, const RopeArgs& a, unsigned grid, cudaStream_t st);  // s2a_rope.cuh

namespace {

constexpr int kWarps = 8;         // as in the kernels
constexpr int kLaneElems = 16;

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
  // A warp each for the groups of rows of all tokens, until the GPU is full; then shares.
  const auto groups_of = [&](uint32_t rows) { return (rows + a.rows_per_warp - 1) / a.rows_per_warp; };
  const auto cut = [&](uint32_t rows, uint32_t ctas, int which) {
    const uint64_t items = tokens * groups_of(rows), warps = (uint64_t)ctas * kWarps;
    a.share[which] = (uint32_t)(items / warps);
    a.more[which] = (uint32_t)(items % warps);
  };
  const auto ctas_for = [&](uint64_t items, uint64_t cap) { return (uint32_t)std::min<uint64_t>((items + kWarps - 1) / kWarps, cap); };
  if (tokens * (groups_of(a.heads[0]) + groups_of(a.heads[1])) >> 32) return cudaErrorInvalidValue;  // more than any memory holds
  unsigned grid;
  if (mode == kRopeBwdNorm) {
    const uint64_t items0 = tokens * groups_of(a.heads[0]), items1 = tokens * groups_of(a.heads[1]);
    const uint64_t cap = 148 * 2, share0 = cap * items0 / (items0 + items1);
    a.ctas0 = items0 ? ctas_for(items0, items1 ? std::min(std::max<uint64_t>(share0, 1), cap - 1) : cap) : 0;
    const uint32_t ctas1 = items1 ? ctas_for(items1, cap - a.ctas0) : 0;
    grid = a.ctas0 + ctas1;
    if (items0) cut(a.heads[0], a.ctas0, 0);
    if (items1) cut(a.heads[1], ctas1, 1);
    a.partials = sums ? scratch : nullptr;
  } else {
    grid = ctas_for(tokens * groups_of(heads), (uint64_t)sm_count() * 3);
    cut(heads, grid, 0);
  }
  // from here on strides are in bytes
  for (HeadsArg* h : {&a.in[0], &a.in[1], &a.grad[0], &a.grad[1], &a.out[0], &a.out[1]}) {
    h->batch *= es;
    h->token *= es;
    h->head *= es;
  }
  const cudaError_t e = dt == kF32 ? launch_rope_kernel<kF32>(mode, V, a, grid, st) : launch_rope_kernel<kBF16>(mode, V, a, grid, st);
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
