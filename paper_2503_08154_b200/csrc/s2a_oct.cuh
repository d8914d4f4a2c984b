// Consecutive elements of an I/O tensor in registers: eight (16 bytes of bfloat16, 32 of binary32), or the piece of 16
// bytes; asynchronous copies, and the launch helpers of the kernels built on them.
#pragma once

#include <atomic>

#include "s2a_common.cuh"

namespace s2a {

template <int DT> struct Eight;
template <> struct Eight<kBF16> {
  uint4 r;
  __device__ __forceinline__ void load(const void* p) { r = *(const uint4*)p; }
  __device__ __forceinline__ void store(void* p) const { *(uint4*)p = r; }
  __device__ __forceinline__ void get(F2* v) const {
    v[0] = f2_from_bf16x2(r.x);
    v[1] = f2_from_bf16x2(r.y);
    v[2] = f2_from_bf16x2(r.z);
    v[3] = f2_from_bf16x2(r.w);
  }
  __device__ __forceinline__ void set(const F2* v) {
    r = make_uint4(f2_to_bf16x2(v[0]), f2_to_bf16x2(v[1]), f2_to_bf16x2(v[2]), f2_to_bf16x2(v[3]));
  }
};
template <> struct Eight<kF32> {
  float4 a, b;
  __device__ __forceinline__ void load(const void* p) { a = ((const float4*)p)[0]; b = ((const float4*)p)[1]; }
  __device__ __forceinline__ void store(void* p) const { ((float4*)p)[0] = a; ((float4*)p)[1] = b; }
  __device__ __forceinline__ void get(F2* v) const {
    v[0] = f2_pack(a.x, a.y);
    v[1] = f2_pack(a.z, a.w);
    v[2] = f2_pack(b.x, b.y);
    v[3] = f2_pack(b.z, b.w);
  }
  __device__ __forceinline__ void set(const F2* v) {
    f2_unpack(v[0], a.x, a.y);
    f2_unpack(v[1], a.z, a.w);
    f2_unpack(v[2], b.x, b.y);
    f2_unpack(v[3], b.z, b.w);
  }
};

template <int DT> constexpr int kVec = DT == kF32 ? 4 : 8;  // elements of a piece: 16 bytes
template <int DT> constexpr int kPairs = kVec<DT> / 2;

// A piece as it lies in memory.
template <int DT>
__device__ __forceinline__ void widen_piece(const uint4& r, F2* v) {
  if constexpr (DT == kF32) {
    v[0] = f2_pack(__uint_as_float(r.x), __uint_as_float(r.y));
    v[1] = f2_pack(__uint_as_float(r.z), __uint_as_float(r.w));
  } else {
    v[0] = f2_from_bf16x2(r.x);
    v[1] = f2_from_bf16x2(r.y);
    v[2] = f2_from_bf16x2(r.z);
    v[3] = f2_from_bf16x2(r.w);
  }
}
template <int DT>
__device__ __forceinline__ uint4 narrow_piece(const F2* v) {
  if constexpr (DT == kF32) {
    float a, b, c, d;
    f2_unpack(v[0], a, b);
    f2_unpack(v[1], c, d);
    return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
  } else {
    return make_uint4(f2_to_bf16x2(v[0]), f2_to_bf16x2(v[1]), f2_to_bf16x2(v[2]), f2_to_bf16x2(v[3]));
  }
}

// One element of a learned parameter (layer norm's weights, a bias table): binary32 or bfloat16 by `wdt`.
__device__ __forceinline__ float load_param(const void* p, uint64_t i, int wdt) {
  return wdt == kF32 ? ((const float*)p)[i] : __bfloat162float(((const __nv_bfloat16*)p)[i]);
}
__device__ __forceinline__ void store_param(void* p, uint64_t i, int wdt, float v) {
  if (wdt == kF32) ((float*)p)[i] = v;
  else ((__nv_bfloat16*)p)[i] = __float2bfloat16_rn(v);
}

// Asynchronous copies of a thread's own pieces into shared memory (16, 8 or 4 bytes, both sides aligned to that), in groups
// that complete in order.  A thread that reads back only what it copied needs no barrier, just the wait.
template <int BYTES>
__device__ __forceinline__ void copy_async(void* smem, const void* global) {
  const uint32_t s = (uint32_t)__cvta_generic_to_shared(smem);
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(s), "l"(global) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(s), "l"(global), "n"(BYTES) : "memory");
}
// The first `bytes` of 16, zeros after them.
__device__ __forceinline__ void copy_async_front(void* smem, const void* global, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(global), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Programmatic dependent launch.  Every kernel launched through launch_overlapped calls enter_grid() before it
// touches memory: the next kernel of the stream may then be scheduled, and this one goes on once its
// predecessor has completed and its writes are visible.
__device__ __forceinline__ void enter_grid() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Lets a kernel use `bytes` of dynamic shared memory on the current device, once per device (`done`: one bit each, a
// static of the caller per kernel; concurrent first calls may both set the attribute).
template <typename... P>
cudaError_t allow_shared(void (*kernel)(P...), size_t bytes, std::atomic<uint64_t>& done) {
  if (bytes <= 40 * 1024) return cudaSuccess;  // within the 48 KB that need no leave, static arrays included
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev < 64 && (done.load(std::memory_order_acquire) & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess && dev < 64) done.fetch_or(bit, std::memory_order_release);
  return e;
}

template <typename... P, typename... A>
cudaError_t launch_overlapped(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

}  // namespace s2a
