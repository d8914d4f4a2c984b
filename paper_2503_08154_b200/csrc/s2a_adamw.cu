// One AdamW step over many tensors, states in 32 bits or in 8, and the norm of all gradients.
//
//   g' = g * scale * factor;  m = m + (1 - b1)(g' - m);  v = b2 v + (1 - b2) g'^2
//   p = p - lr * wd * p - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// 8-bit states: e4m3 codes of m and of sqrt(v) (the root has half of v's range of exponents, and the step needs the root), 448
// standing for the largest magnitude of a block of 256 elements, which is kept in 32 bits.  A root above zero never gets
// the code zero: an m over a root that was rounded away would be a step of m / eps.  Rounded to nearest, a state that moves by
// less than half a step of its code a step stays where it is (with b2 = 0.999 sqrt(v) moves by 0.05 %, a code's step is 6 to 12 %);
// rounded at random, by the 16 bits of a counter-based generator, it moves as it should on average.
//
// Bound by memory: a warp takes 256 elements at a time, eight neighbouring ones a lane, everything of them in registers between
// one load and one store, the block's largest magnitudes by two warp reductions.  A chunk of four such blocks is what a warp takes from the
// plan at a time; the plan has the tensor of each chunk, so that no warp searches.
#include "s2a_launch.h"
#include "s2a_oct.cuh"
#include "s2a_philox.cuh"

namespace s2a {
namespace {

constexpr int kStepWarps = 8;
constexpr int kStepThreads = kStepWarps * 32;
constexpr float kTopCode = 448.0f;          // the largest e4m3 value
constexpr uint32_t kTopBits = 0x7Eu;        // and its code
constexpr float kTwoM120 = 7.52316384526264e-37f, kTwo120 = 1.329227995784916e+36f;

// Eight neighbouring elements: `count` of them exist.  `vec`: they lie on the 16-byte grid.
template <int DT>
__device__ __forceinline__ void load8(const void* base, uint64_t at, uint32_t count, bool vec, float (&f)[8]) {
  const typename Io<DT>::T* p = (const typename Io<DT>::T*)base + at;
  if (vec && count == 8) {
    if constexpr (DT == kF32) {
      const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
      f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
    } else {
      const uint4 r = *(const uint4*)p;
      const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (uint32_t)i < count ? Io<DT>::widen(p[i]) : 0.0f;
  }
}

template <int DT>
__device__ __forceinline__ void store8(void* base, uint64_t at, uint32_t count, bool vec, const float (&f)[8]) {
  typename Io<DT>::T* p = (typename Io<DT>::T*)base + at;
  if (vec && count == 8) {
    if constexpr (DT == kF32) {
      ((float4*)p)[0] = make_float4(f[0], f[1], f[2], f[3]);
      ((float4*)p)[1] = make_float4(f[4], f[5], f[6], f[7]);
    } else {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = f2_to_bf16x2(f2_pack(f[2 * i], f[2 * i + 1]));
      *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((uint32_t)i < count) p[i] = Io<DT>::narrow(f[i]);
  }
}

__device__ __forceinline__ void load_codes(const void* base, uint64_t at, uint32_t count, bool vec, uint32_t (&w)[2]) {
  const uint8_t* p = (const uint8_t*)base + at;
  if (vec && count == 8) {
    const uint2 r = *(const uint2*)p;
    w[0] = r.x;
    w[1] = r.y;
  } else {
    w[0] = w[1] = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((uint32_t)i < count) w[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
  }
}
__device__ __forceinline__ void store_codes(void* base, uint64_t at, uint32_t count, bool vec, const uint32_t (&w)[2]) {
  uint8_t* p = (uint8_t*)base + at;
  if (vec && count == 8) {
    *(uint2*)p = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((uint32_t)i < count) p[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

// The value of an e4m3 code: times 2^-120 the type's exponents are those of binary32, its subnormals too.  (The codes 0x7F and
// 0xFF, which nothing here writes, come out as 480.)
__device__ __forceinline__ float code_value(uint32_t code) {
  return __uint_as_float(((code & 0x7Fu) << 20) | ((code & 0x80u) << 24)) * kTwo120;
}
// The code of a magnitude x of at most 448: to nearest (ties to even), or with 16 random bits, and half of one, below the last kept bit.
__device__ __forceinline__ uint32_t code_of(float x, bool random, uint32_t bits) {
  const uint32_t w = __float_as_uint(x * kTwoM120);
  const uint32_t add = random ? (bits << 4) | 8u : 0x7FFFFu + ((w >> 20) & 1u);
  const uint32_t code = (w + add) >> 20;
  return code < kTopBits ? code : kTopBits;
}

__device__ __forceinline__ float approx_sqrt(float x) {
  float y;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// What is the same for every element of a step.
struct Rates {
  float scale, lr, first, root;  // lr / (1 - b1^t) and 1 / sqrt(1 - b2^t)
  uint64_t count;                // the generator's second counter word
};

// bfloat16 at random: 16 random bits below the last kept one.  An infinity stays one; a NaN too.
__device__ __forceinline__ float random_bf16(float x, uint32_t bits) {
  const uint32_t w = __float_as_uint(x);
  if ((w & 0x7F800000u) == 0x7F800000u) return x;
  return __uint_as_float((w + bits) & 0xFFFF0000u);
}

// One block of 256 elements (or the `count` elements of a lane that exist).
template <int PDT, int GDT, int BITS, bool RANDOM>
__device__ __forceinline__ void step_block(const StepArgs& a, const StepTensor& t, const Rates& r, const PhiloxKey& key, uint64_t draw,
                                           uint64_t at, uint32_t count, bool vec, uint64_t block) {
  const uint32_t lane = threadIdx.x & 31u;
  float p[8], g[8], m[8], v[8], root[8];
  load8<GDT>(t.g, at, count, vec, g);
  load8<PDT>(t.p, at, count, vec, p);
  if constexpr (BITS == 32) {
    load8<kF32>(t.m, at, count, vec, m);
    load8<kF32>(t.v, at, count, vec, v);
  } else {
    uint32_t mw[2], vw[2];
    load_codes(t.m, at, count, vec, mw);
    load_codes(t.v, at, count, vec, vw);
    const float ms = t.m_scale[block] * (1.0f / kTopCode), vs = t.v_scale[block] * (1.0f / kTopCode);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m[i] = code_value((mw[i / 4] >> (8 * (i % 4))) & 0xFFu) * ms;
      const float x = code_value((vw[i / 4] >> (8 * (i % 4))) & 0x7Fu) * vs;
      v[i] = x * x;
    }
  }
  const float shrink = r.lr * t.decay * t.lr, step = r.first * t.lr;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = g[i] * r.scale;
    m[i] = fmaf(a.one_beta1, x - m[i], m[i]);
    v[i] = fmaf(a.one_beta2 * x, x, a.beta2 * v[i]);
    root[i] = approx_sqrt(v[i]);
    p[i] = fmaf(-shrink, p[i], p[i]) - __fdividef(step * m[i], fmaf(root[i], r.root, a.eps));
  }
  if (PDT == kBF16 && RANDOM) {
    float q[8];
    const uint4 bits = philox(key, (draw + lane) | (1ull << 63), r.count);
    const uint32_t w[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = random_bf16(p[i], i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu);
    store8<PDT>(t.p, at, count, vec, q);
  } else {
    store8<PDT>(t.p, at, count, vec, p);
  }
  if (PDT == kF32 && t.copy) store8<kBF16>(t.copy, at, count, vec, p);
  if constexpr (BITS == 32) {
    store8<kF32>(t.m, at, count, vec, m);
    store8<kF32>(t.v, at, count, vec, v);
  } else {
    // magnitudes as whole numbers: a NaN is above everything and makes the block's scale one
    uint32_t tm = 0u, tv = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if ((uint32_t)i >= count) m[i] = root[i] = 0.0f;
      tm = max(tm, __float_as_uint(m[i]) & 0x7FFFFFFFu);
      tv = max(tv, __float_as_uint(root[i]) & 0x7FFFFFFFu);
    }
    const float top_m = __uint_as_float(__reduce_max_sync(0xffffffffu, tm)), top_v = __uint_as_float(__reduce_max_sync(0xffffffffu, tv));
    // a block whose largest magnitude is below 2^-110 is stored as zeros
    const float im = top_m >= 7.703719777548943e-34f ? __fdiv_rn(kTopCode, top_m) : 0.0f;
    const float iv = top_v >= 7.703719777548943e-34f ? __fdiv_rn(kTopCode, top_v) : 0.0f;
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    if (RANDOM) {
      const uint4 bits = philox(key, draw + lane, r.count);
      w[0] = bits.x, w[1] = bits.y, w[2] = bits.z, w[3] = bits.w;
    }
    uint32_t mw[2] = {0u, 0u}, vw[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t bits = i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xFFFFu;
      const uint32_t other = __byte_perm(bits, 0u, 0x4401);  // the root's: the two bytes the other way round
      uint32_t c = code_of(fabsf(m[i]) * im, RANDOM, bits) | (m[i] < 0.0f ? 0x80u : 0u);
      mw[i / 4] |= c << (8 * (i % 4));
      c = code_of(root[i] * iv, RANDOM, other);
      if (c == 0u && root[i] * iv > 0.0f) c = 1u;
      vw[i / 4] |= c << (8 * (i % 4));
    }
    store_codes(t.m, at, count, vec, mw);
    store_codes(t.v, at, count, vec, vw);
    if (lane == 0) {
      t.m_scale[block] = top_m;
      t.v_scale[block] = top_v;
    }
  }
}

template <int PDT, int GDT, int BITS, bool RANDOM>
__global__ void __launch_bounds__(kStepThreads) adamw_kernel(StepArgs a) {
  enter_grid();
  const uint32_t lane = threadIdx.x & 31u;
  Rates r;
  r.scale = a.control[2];
  r.lr = a.control[0];
  if (a.clip) {
    const float norm = a.clip[0];
    if (!(fabsf(norm) <= 3.4028235e38f)) return;  // gradients that overflowed: nothing is changed
    r.scale *= a.clip[1];
  }
  const float number = a.control[1];
  r.first = __fdiv_rn(r.lr, -expm1f(number * a.log_beta1));
  r.root = __frsqrt_rn(-expm1f(number * a.log_beta2));
  const PhiloxKey key(RANDOM ? a.rng[0] : 0ull);
  r.count = RANDOM ? a.rng[1] + a.site : 0ull;
  for (uint64_t c = (uint64_t)blockIdx.x * kStepWarps + (threadIdx.x >> 5); c < a.n_chunks; c += (uint64_t)gridDim.x * kStepWarps) {
    const StepTensor t = a.tensors[a.owner[c]];
    const uint64_t from = (c - t.chunk0) * kStepChunk;
    // random bits and blocks are counted from the tensor's first element, and its vectors with them
    constexpr bool COUNTED = RANDOM || BITS == 8;
    const bool vec = COUNTED ? t.head == 0u : t.head != kStepScalar;
    const uint32_t head = vec ? t.head : 0u;
    // the elements before the grid, as a block of one lane's
    if (!COUNTED && head && from == 0)
      step_block<PDT, GDT, BITS, RANDOM>(a, t, r, key, t.block0 * 32, 0, lane == 0 ? (t.n < head ? (uint32_t)t.n : head) : 0u, false, 0);
#pragma unroll 1
    for (uint32_t k = 0; k < kStepChunk / kStepBlock; ++k) {
      const uint64_t base = head + from + k * kStepBlock;
      if (base >= t.n) break;
      const uint64_t at = base + 8 * lane, block = (from + k * kStepBlock) / kStepBlock;
      const uint32_t count = at >= t.n ? 0u : (t.n - at < 8 ? (uint32_t)(t.n - at) : 8u);
      step_block<PDT, GDT, BITS, RANDOM>(a, t, r, key, (t.block0 + block) * 32, at, count, vec, block);
    }
  }
}

// ---------------------------------------------------------------- the gradients' norm
// Squares of eight elements: in 32 bits where the largest magnitude is from 2^-40 to 2^50, whose squares neither overflow nor, beside
// it, vanish; else in 64.  Sums of eights are added in 64 bits.
template <int GDT>
__device__ __forceinline__ double square_sum(const float (&g)[8]) {
  float top = 0.0f, s = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    top = fmaxf(top, fabsf(g[i]));
    s = fmaf(g[i], g[i], s);
  }
  if (top == 0.0f || (top >= 9.094947e-13f && top <= 1.1258999e15f)) return (double)s;
  double d = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) d = fma((double)g[i], (double)g[i], d);
  return d;
}

template <int GDT>
__global__ void __launch_bounds__(kStepThreads) grad_norm_kernel(StepArgs a, double* partials) {
  __shared__ double buf[kStepWarps];
  enter_grid();
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  double sum = 0.0;
  for (uint64_t c = (uint64_t)blockIdx.x * kStepWarps + warp; c < a.n_chunks; c += (uint64_t)gridDim.x * kStepWarps) {
    const StepTensor t = a.tensors[a.owner[c]];
    const uint64_t from = (c - t.chunk0) * kStepChunk;
    const bool vec = t.head != kStepScalar;
    const uint32_t head = vec ? t.head : 0u;
    float g[8];
    if (head && from == 0) {
      load8<GDT>(t.g, 0, lane == 0 ? (t.n < head ? (uint32_t)t.n : head) : 0u, false, g);
      sum += square_sum<GDT>(g);
    }
#pragma unroll
    for (uint32_t k = 0; k < kStepChunk / kStepBlock; ++k) {
      const uint64_t at = head + from + k * kStepBlock + 8 * lane;
      const uint32_t count = at >= t.n ? 0u : (t.n - at < 8 ? (uint32_t)(t.n - at) : 8u);
      load8<GDT>(t.g, at, count, vec, g);
      sum += square_sum<GDT>(g);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) buf[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kStepWarps; ++w) sum += buf[w];
    partials[blockIdx.x] = sum;
  }
}

__global__ void __launch_bounds__(1024) grad_norm_finish_kernel(const double* partials, uint32_t n, const float* control, float max_norm,
                                                                float* out) {
  __shared__ double buf[32];
  enter_grid();
  double sum = 0.0;
  for (uint32_t i = threadIdx.x; i < n; i += 1024) sum += partials[i];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (threadIdx.x % 32 == 0) buf[threadIdx.x / 32] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < 32; ++w) sum += buf[w];
    const double norm = sqrt(sum) * fabs((double)control[2]);
    const double factor = (double)max_norm / (norm + 1e-6);
    out[0] = (float)norm;
    out[1] = (float)(factor > 1.0 ? 1.0 : factor);
  }
}

template <int PDT, int GDT>
cudaError_t launch_adamw_types(int bits, const StepArgs& a, unsigned grid, cudaStream_t st) {
  if (bits == 32)
    return a.rng ? launch_overlapped(adamw_kernel<PDT, GDT, 32, true>, dim3(grid), kStepThreads, 0, st, a)
                 : launch_overlapped(adamw_kernel<PDT, GDT, 32, false>, dim3(grid), kStepThreads, 0, st, a);
  return a.rng ? launch_overlapped(adamw_kernel<PDT, GDT, 8, true>, dim3(grid), kStepThreads, 0, st, a)
               : launch_overlapped(adamw_kernel<PDT, GDT, 8, false>, dim3(grid), kStepThreads, 0, st, a);
}

}  // namespace

cudaError_t launch_adamw(int pdt, int gdt, int state_bits, const StepArgs& a, cudaStream_t st) {
  if (a.n_chunks == 0) return cudaSuccess;
  const uint64_t want = ((uint64_t)a.n_chunks + kStepWarps - 1) / kStepWarps, cap = (uint64_t)sm_count() * 16;
  const unsigned grid = (unsigned)(want < cap ? want : cap);
  if (pdt == kF32)
    return gdt == kF32 ? launch_adamw_types<kF32, kF32>(state_bits, a, grid, st) : launch_adamw_types<kF32, kBF16>(state_bits, a, grid, st);
  return gdt == kF32 ? launch_adamw_types<kBF16, kF32>(state_bits, a, grid, st) : launch_adamw_types<kBF16, kBF16>(state_bits, a, grid, st);
}

uint64_t grad_norm_scratch_bytes(uint32_t n_chunks) {
  const uint64_t want = ((uint64_t)n_chunks + kStepWarps - 1) / kStepWarps;
  return (want < 1 ? 1 : (want < kMaxNormCtas ? want : kMaxNormCtas)) * sizeof(double);
}

cudaError_t launch_grad_norm(int gdt, const StepArgs& a, float max_norm, float* out, double* scratch, cudaStream_t st) {
  const unsigned grid = (unsigned)(grad_norm_scratch_bytes(a.n_chunks) / sizeof(double));
  const cudaError_t e = gdt == kF32 ? launch_overlapped(grad_norm_kernel<kF32>, dim3(grid), kStepThreads, 0, st, a, scratch)
                                    : launch_overlapped(grad_norm_kernel<kBF16>, dim3(grid), kStepThreads, 0, st, a, scratch);
  if (e != cudaSuccess) return e;
  return launch_overlapped(grad_norm_finish_kernel, dim3(1), 1024, 0, st, (const double*)scratch, grid, a.control, max_norm, out);
}

}  // namespace s2a
