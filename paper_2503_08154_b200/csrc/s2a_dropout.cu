// Dropout whose mask is never stored: forward and backward draw the same bits from a counter-based generator.
//
// Element e of a call owns the 16-bit field e mod 8 of Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel
// random numbers: as easy as 1, 2, 3", SC 2011) at counter (e / 8, offset + site) under the 64-bit key `seed`: word
// w holds elements 2w (low half) and 2w + 1 (high half).  One evaluation serves the eight elements of a 16-byte
// bfloat16 vector.  Sixteen bits an element, not thirty-two:
// with two evaluations for eight elements the kernel is bound by the generator's multiplications, and 200,000,003 bfloat16
// elements take 176 us instead of 126.
#include "s2a_launch.h"
#include "s2a_oct.cuh"

namespace s2a {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 2;          // vectors of a thread in flight
constexpr int kResident = 5;       // CTAs of an SM
// Four times as many CTAs as fit: the last ones even out what the SMs have left.  [200,000,003] bfloat16: 126 us (6.34 TB/s; in long
// runs, at lower clocks, up to 138 us), against 132 with exactly as many as fit, and 154 with one vector in flight; [64, 12, 197, 197]:
// 21.4, 21.7, 25.1 us.
constexpr int kCtasPerSm = 20;

struct PhiloxKey {
  uint32_t k0[10], k1[10];
  __device__ __forceinline__ explicit PhiloxKey(uint64_t seed) {
    uint32_t a = (uint32_t)seed, b = (uint32_t)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
      k0[i] = a;
      k1[i] = b;
      a += 0x9E3779B9u;
      b += 0xBB67AE85u;
    }
  }
};

__device__ __forceinline__ uint4 philox(const PhiloxKey& key, uint64_t block, uint64_t count) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)count, c3 = (uint32_t)(count >> 32);
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(p1 >> 32) ^ c1 ^ key.k0[i];
    c1 = (uint32_t)p1;
    c2 = (uint32_t)(p0 >> 32) ^ c3 ^ key.k1[i];
    c3 = (uint32_t)p0;
  }
  return make_uint4(c0, c1, c2, c3);
}

// An element is kept when its 16 bits are at least T; `limit` is T << 16, so that each field is compared in the
// top half of a word, and what lies below it does not matter.
__device__ __forceinline__ F2 keep_pair(F2 v, uint32_t word, uint32_t limit) {
  float lo, hi;
  f2_unpack(v, lo, hi);
  return f2_pack((word << 16) >= limit ? lo : 0.0f, word >= limit ? hi : 0.0f);
}

// in = x (forward) or grad_out (backward).  A dropped element is selected away, not multiplied by zero, so that an
// infinity or a NaN in its place leaves no trace.  RES: y = residual + dropout(x), the product and the sum in one
// rounding (fma).
template <int DT, bool RES>
__device__ __forceinline__ void apply(Eight<DT>& v, const Eight<DT>& r, const uint4& bits, uint32_t limit, F2 scale) {
  F2 a[4], b[4];
  v.get(a);
  if (RES) r.get(b);
  const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    a[k] = keep_pair(a[k], w[k], limit);
    a[k] = RES ? f2_fma(a[k], scale, b[k]) : f2_mul(a[k], scale);
  }
  v.set(a);
}

template <int DT, bool RES>
__global__ void __launch_bounds__(kThreads, kResident) dropout_kernel(const void* xv, const void* rv, void* yv, uint64_t n,
                                                           const uint64_t* rng, uint64_t site, uint32_t limit, float scale) {
  using T = typename Io<DT>::T;
  enter_grid();
  const T* x = (const T*)xv;
  const T* res = (const T*)rv;
  T* y = (T*)yv;
  const PhiloxKey key(rng[0]);
  const uint64_t count = rng[1] + site;
  const F2 scale2 = f2_both(scale);
  const uint64_t n8 = n >> 3, stride = (uint64_t)gridDim.x * kThreads;
  uint64_t b = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
#pragma unroll 1
  for (; b + (kAhead - 1) * stride < n8; b += kAhead * stride) {
    Eight<DT> v[kAhead], r[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      v[k].load(x + 8 * (b + k * stride));
      if (RES) r[k].load(res + 8 * (b + k * stride));
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      apply<DT, RES>(v[k], r[k], philox(key, b + k * stride, count), limit, scale2);
      v[k].store(y + 8 * (b + k * stride));
    }
  }
  for (; b < n8; b += stride) {
    Eight<DT> v, r;
    v.load(x + 8 * b);
    if (RES) r.load(res + 8 * b);
    apply<DT, RES>(v, r, philox(key, b, count), limit, scale2);
    v.store(y + 8 * b);
  }
  if (blockIdx.x == 0 && threadIdx.x < (n & 7u)) {  // the last, partial eight: an element a thread
    const uint64_t e = 8 * n8 + threadIdx.x;
    const uint4 bits = philox(key, n8, count);
    const uint32_t word = threadIdx.x < 2 ? bits.x : (threadIdx.x < 4 ? bits.y : (threadIdx.x < 6 ? bits.z : bits.w));
    const uint32_t field = (threadIdx.x & 1u) ? word : word << 16;
    const float v = field >= limit ? Io<DT>::widen(x[e]) : 0.0f;
    y[e] = Io<DT>::narrow(RES ? __fmaf_rn(v, scale, Io<DT>::widen(res[e])) : __fmul_rn(v, scale));
  }
}

}  // namespace

cudaError_t launch_dropout(int dt, const void* x, const void* residual, void* y, uint64_t n, const uint64_t* rng,
                           uint64_t site, uint32_t threshold, cudaStream_t st) {
  if (n == 0) return cudaSuccess;
  if (threshold >= 65536u) {  // everything is dropped: the residual alone, or zeros
    const size_t bytes = n * (dt == kF32 ? 4u : 2u);
    if (!residual) return cudaMemsetAsync(y, 0, bytes, st);
    return y == residual ? cudaSuccess : cudaMemcpyAsync(y, residual, bytes, cudaMemcpyDeviceToDevice, st);
  }
  const uint64_t want = ((n >> 3) + kThreads - 1) / kThreads, cap = (uint64_t)sm_count() * kCtasPerSm;
  const dim3 grid((unsigned)(want < 1 ? 1 : (want < cap ? want : cap)));
  const float scale = (float)(65536.0 / (65536.0 - threshold));
  const uint32_t limit = threshold << 16;
  if (dt == kF32)
    return residual ? launch_overlapped(dropout_kernel<kF32, true>, grid, kThreads, 0, st, x, residual, y, n, rng, site, limit, scale)
                    : launch_overlapped(dropout_kernel<kF32, false>, grid, kThreads, 0, st, x, residual, y, n, rng, site, limit, scale);
  return residual ? launch_overlapped(dropout_kernel<kBF16, true>, grid, kThreads, 0, st, x, residual, y, n, rng, site, limit, scale)
                  : launch_overlapped(dropout_kernel<kBF16, false>, grid, kThreads, 0, st, x, residual, y, n, rng, site, limit, scale);
}

}  // namespace s2a
