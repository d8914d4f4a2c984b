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
// A warp takes 256 elements at a time, eight neighbouring ones a lane, everything of them in registers between
// one load and one store, the block's largest magnitudes by two warp reductions.  What a warp takes from the plan
// at a time is a chunk of such blocks; the plan has the tensor of each chunk, so that no warp searches.  32-bit states are bound by
// memory (302 M weights with bfloat16 gradients and copies 1.30 ms, a copy's rate); 8-bit states rounded at random by
// the instructions of the formula step by step, rounding and generator, some 460 a block and warp: the same weights in bfloat16 take 684 us
// (0.68 of a copy's rate) in runs of some ms, and 750 (0.62) in longer ones, in which the power limit takes the clock from 1.97 to 1.78 GHz.
#include "s2a_launch.h"
#include "s2a_oct.cuh"
#include "s2a_philox.cuh"

namespace s2a {
namespace {

constexpr int kStepWarps = 4;
constexpr int kStepThreads = kStepWarps * 32;
constexpr int kNormWarps = 8;
constexpr int kNormThreads = kNormWarps * 32;
constexpr float kTopCode = 448.0f;                // the largest e4m3 value
constexpr float kTwoM120 = 7.52316384526264e-37f;
constexpr float kTwoM64 = 5.421010862427522e-20f;
constexpr float kSmallest = 7.703719777548943e-34f;  // 2^-110: a block of which the largest magnitude is below is stored as zeros

// A lane's eight elements of a block.  QUAD: elements 4 lane .. 4 lane + 3 and 128 more, so that a warp's accesses of binary32 have no gaps;
// otherwise 8 lane .. 8 lane + 7, which share 128 random bits.  `first` and `left`: where its elements begin and how many of the
// tensor's there are from there on.
// WHOLE: the block is, and on the 16-byte grid.
template <bool QUAD, bool WHOLE = false>
struct Spot {
  uint64_t first;
  int32_t left;  // from `first`, at most 256
  __device__ __forceinline__ int32_t count(int half) const {  // of the four elements of a half
    if (WHOLE) return 4;
    const int32_t n = left - (QUAD ? 128 : 4) * half;
    return n < 0 ? 0 : (n < 4 ? n : 4);
  }
  __device__ __forceinline__ uint64_t at(int half) const { return first + (QUAD ? 128 : 4) * half; }
};

// Eight elements as they lie in memory: binary32 in eight words, bfloat16 in four, codes in two.
template <int ES>
struct Raw {
  uint32_t w[2 * ES];
  template <bool QUAD, bool WHOLE>
  __device__ __forceinline__ void load(const void* base, const Spot<QUAD, WHOLE>& s, bool vec) {
    const char* p = (const char*)base;
    if (WHOLE || (vec && s.count(1) == 4)) {  // all eight
      if constexpr (ES == 4) {
        const uint4 a = *(const uint4*)(p + s.at(0) * 4), b = *(const uint4*)(p + s.at(1) * 4);
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
      } else if constexpr (ES == 2 && !QUAD) {
        const uint4 a = *(const uint4*)(p + s.at(0) * 2);
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
      } else if constexpr (ES == 2) {
        const uint2 a = *(const uint2*)(p + s.at(0) * 2), b = *(const uint2*)(p + s.at(1) * 2);
        w[0] = a.x, w[1] = a.y, w[2] = b.x, w[3] = b.y;
      } else {
        const uint2 a = *(const uint2*)(p + s.at(0));
        w[0] = a.x, w[1] = a.y;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2 * ES; ++i) w[i] = 0u;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i % 4 < s.count(i / 4)) {
          const uint64_t at = s.at(i / 4) + i % 4;
          if constexpr (ES == 4) w[i] = ((const uint32_t*)base)[at];
          else if constexpr (ES == 2) w[i / 2] |= (uint32_t)((const uint16_t*)base)[at] << (16 * (i % 2));
          else w[i / 4] |= (uint32_t)((const uint8_t*)base)[at] << (8 * (i % 4));
        }
    }
  }
  template <bool QUAD, bool WHOLE>
  __device__ __forceinline__ void store(void* base, const Spot<QUAD, WHOLE>& s, bool vec) const {
    char* p = (char*)base;
    if (WHOLE || (vec && s.count(1) == 4)) {
      if constexpr (ES == 4) {
        *(uint4*)(p + s.at(0) * 4) = make_uint4(w[0], w[1], w[2], w[3]);
        *(uint4*)(p + s.at(1) * 4) = make_uint4(w[4], w[5], w[6], w[7]);
      } else if constexpr (ES == 2 && !QUAD) {
        *(uint4*)(p + s.at(0) * 2) = make_uint4(w[0], w[1], w[2], w[3]);
      } else if constexpr (ES == 2) {
        *(uint2*)(p + s.at(0) * 2) = make_uint2(w[0], w[1]);
        *(uint2*)(p + s.at(1) * 2) = make_uint2(w[2], w[3]);
      } else {
        *(uint2*)(p + s.at(0)) = make_uint2(w[0], w[1]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i % 4 < s.count(i / 4)) {
          const uint64_t at = s.at(i / 4) + i % 4;
          if constexpr (ES == 4) ((uint32_t*)base)[at] = w[i];
          else if constexpr (ES == 2) ((uint16_t*)base)[at] = (uint16_t)(w[i / 2] >> (16 * (i % 2)));
          else ((uint8_t*)base)[at] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
        }
    }
  }
  // as binary32, two by two (elements; codes: their values)
  __device__ __forceinline__ void get(F2 (&f)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (ES == 4) f[i] = f2_pack(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
      else if constexpr (ES == 2) f[i] = f2_from_bf16x2(w[i]);
      else f[i] = code_values((uint16_t)(w[i / 2] >> (16 * (i % 2))));
    }
  }
  __device__ __forceinline__ void set(const F2 (&f)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (ES == 4) {
        float a, b;
        f2_unpack(f[i], a, b);
        w[2 * i] = __float_as_uint(a);
        w[2 * i + 1] = __float_as_uint(b);
      } else {
        static_assert(ES == 2, "codes are put together elsewhere");
        w[i] = f2_to_bf16x2(f[i]);
      }
    }
  }
  // two e4m3 codes, each exactly a binary16 number
  static __device__ __forceinline__ F2 code_values(uint16_t codes) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(codes));
    float lo, hi;
    asm("{.reg .b16 a, b; mov.b32 {a, b}, %2; cvt.f32.f16 %0, a; cvt.f32.f16 %1, b;}" : "=f"(lo), "=f"(hi) : "r"(h));
    return f2_pack(lo, hi);
  }
};

// One step of binary32 at most; what is below the normal range counts as zero, which saves the instructions of its scaling.
__device__ __forceinline__ float approx_sqrt(float x) {
  float y;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The round keys of the generator, from shared memory: in registers all twenty would cost the kernel a CTA of each SM.
struct SharedKey {
  const uint4* keys;  // of two rounds each
  __device__ __forceinline__ uint4 draw(uint64_t block, uint64_t count) const {
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)count, c3 = (uint32_t)(count >> 32);
#pragma unroll
    for (int i = 0; i < 5; ++i) {
      const uint4 k = keys[i];
      philox_round(c0, c1, c2, c3, k.x, k.y);
      philox_round(c0, c1, c2, c3, k.z, k.w);
    }
    return make_uint4(c0, c1, c2, c3);
  }
};

// What is the same for every element of a step.
struct Rates {
  float lr, first, root;   // lr / (1 - b1^t) and 1 / sqrt(1 - b2^t)
  float grad1, grad2;      // 32-bit states: what a gradient is multiplied with for m, and for sqrt(v): scale (1 - b1), scale sqrt(1 - b2)
  float scale, one1, one2, beta2;  // 8-bit states: the gradients' scale, 1 - b1, 1 - b2, b2
  uint64_t count;          // the generator's second counter word
};

// Sum and difference of two pairs, each rounded: packed, ptxas would join them with the products before them.
__device__ __forceinline__ F2 add_rounded(F2 a, F2 b) {
  float x, y, u, v;
  f2_unpack(a, x, y);
  f2_unpack(b, u, v);
  return f2_pack(__fadd_rn(x, u), __fadd_rn(y, v));
}
__device__ __forceinline__ F2 sub_rounded(F2 a, F2 b) {
  float x, y, u, v;
  f2_unpack(a, x, y);
  f2_unpack(b, u, v);
  return f2_pack(__fsub_rn(x, u), __fsub_rn(y, v));
}

// The rounded roots of two numbers: v times the approximate reciprocal root, and one step of Newton's iteration on the remainder (Markstein, "Computation
// of elementary functions on the IBM RISC System/6000 processor", 1990); with __fsqrt_rn the codes of 302 M weights are the same, and the step that rounds at
// random takes 4 % longer.  The iteration makes NaN of infinities and of zeros (what is below the normal range among them); v 2^-64, which is never
// above the root, takes their place.
__device__ __forceinline__ F2 roots(F2 v) {
  float x, y, u, w;
  f2_unpack(v, x, y);
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(u) : "f"(x));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(y));
  const F2 q = f2_pack(u, w), s = f2_mul(v, q);
  const F2 r = f2_fma(f2_fma(f2_mul(s, f2_both(-1.0f)), s, v), f2_mul(q, f2_both(0.5f)), s);
  f2_unpack(r, x, y);
  f2_unpack(f2_mul(v, f2_both(kTwoM64)), u, w);
  return f2_pack(fmaxf(x, u), fmaxf(y, w));
}

// 8-bit states: m' and sqrt(v') from the gradients and the codes of m and sqrt(v); unit_m and unit_v are what a code counts.
//   m' = m + (1 - b1)(g' - m),  v' = b2 v + ((1 - b2) g') g'
// Each operation is rounded to binary32, in this order.  Codes come back in the next step: one that a last bit puts on the other side of a border between
// codes is off by 6 to 12 % from there on, and with it the weight and, where it becomes the largest, its block's scale.  So the codes are those of the
// formula as it stands, bit for bit.  (With the factors folded into fused products and an approximate root, 1.2 codes of a million came out as
// the neighbour's, as near to the exact state on average; 302 M weights rounded at random took 608 us in place of 684.)
__device__ __forceinline__ void moments(const F2 (&g)[4], F2 (&m)[4], F2 (&r)[4], const Rates& k, float unit_m, float unit_v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const F2 s = f2_mul(g[i], f2_both(k.scale)), o = f2_mul(m[i], f2_both(unit_m)), q = f2_mul(r[i], f2_both(unit_v));
    m[i] = add_rounded(o, f2_mul(sub_rounded(s, o), f2_both(k.one1)));
    r[i] = roots(add_rounded(f2_mul(f2_mul(q, q), f2_both(k.beta2)), f2_mul(f2_mul(s, f2_both(k.one2)), s)));
  }
}

// p' = p - shrink p - step m / (root sqrt(v) + eps)
__device__ __forceinline__ void update(F2 (&p)[4], const F2 (&m)[4], const F2 (&r)[4], float shrink, float step, float root, float eps) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x, y;
    f2_unpack(f2_fma(r[i], f2_both(root), f2_both(eps)), x, y);
    const F2 q = f2_mul(m[i], f2_pack(rcp_approx(x), rcp_approx(y)));
    p[i] = f2_fma(q, f2_both(-step), f2_fma(p[i], f2_both(-shrink), p[i]));
  }
}

// bfloat16 at random: 16 random bits below the last kept one; an infinity or a NaN stays what it is.
__device__ __forceinline__ void random_bf16(const F2 (&p)[4], const uint4& bits, Raw<2>& out) {
  const uint32_t b[4] = {bits.x, bits.y, bits.z, bits.w};
  F2 zero = f2_both(0.0f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    zero = f2_fma(p[i], f2_both(0.0f), zero);  // NaN once one is not finite
    float x, y;
    f2_unpack(p[i], x, y);
    out.w[i] = __byte_perm(__float_as_uint(x) + (b[i] & 0xFFFFu), __float_as_uint(y) + (b[i] >> 16), 0x7632);
  }
  float x, y;
  f2_unpack(zero, x, y);
  if (!(x + y == 0.0f)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f2_unpack(p[i], x, y);
      if (!(fabsf(x) <= 3.4028235e38f)) out.w[i] = (out.w[i] & 0xFFFF0000u) | (f2_to_bf16x2(f2_pack(x, 0.0f)) & 0xFFFFu);
      if (!(fabsf(y) <= 3.4028235e38f)) out.w[i] = (out.w[i] & 0x0000FFFFu) | (f2_to_bf16x2(f2_pack(0.0f, y)) & 0xFFFF0000u);
    }
  }
}

// The e4m3 codes of eight values x / scale * 448, |x| at most the scale, with 16 random bits and half of one below the last kept bit.
// Times 2^-120 (LARGE: apart from `inverse`, which would leave the normal range) the type's exponents are those of binary32, its subnormals too:
// a code is what stands from bit 20 on, moved to bit 24 here, so that a code is a byte and each field of random bits lies where one byte permutation puts it.  (The
// largest is at most three roundings above 448, and with the bits below the code at most 0xFFFF80 cannot carry.)  SIGNED: m; otherwise sqrt(v),
// whose fields have their bytes exchanged and which is never rounded from above zero to zero.
template <bool SIGNED, bool LARGE>
__device__ __forceinline__ void random_codes(const F2 (&x)[4], float inverse, const uint4& bits, Raw<1>& out) {
  const uint32_t b[4] = {bits.x, bits.y, bits.z, bits.w};
  uint32_t c[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo, hi;
    f2_unpack(LARGE ? f2_mul(f2_mul(x[i], f2_both(inverse)), f2_both(kTwoM120)) : f2_mul(x[i], f2_both(inverse)), lo, hi);
    c[2 * i] = (__float_as_uint(lo) << 4) + __byte_perm(b[i], 0x80u, SIGNED ? 0x5104 : 0x5014);
    c[2 * i + 1] = (__float_as_uint(hi) << 4) + __byte_perm(b[i], 0x80u, SIGNED ? 0x5324 : 0x5234);
    if (SIGNED) {
      f2_unpack(x[i], lo, hi);
      c[2 * i] = (c[2 * i] & 0x7FFFFFFFu) | (__float_as_uint(lo) & 0x80000000u);
      c[2 * i + 1] = (c[2 * i + 1] & 0x7FFFFFFFu) | (__float_as_uint(hi) & 0x80000000u);
    }
  }
  if (!SIGNED) {
    const uint32_t least = __vimin3_u32(__vimin3_u32(c[0], c[1], c[2]), __vimin3_u32(c[3], c[4], c[5]), min(c[6], c[7]));
    if (least < 0x01000000u) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float lo, hi;
        f2_unpack(x[i / 2], lo, hi);
        if (c[i] < 0x01000000u && (i % 2 ? hi : lo) > 0.0f && inverse > 0.0f) c[i] = 0x01000000u;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
    out.w[i] = __byte_perm(__byte_perm(c[4 * i], c[4 * i + 1], 0x0073), __byte_perm(c[4 * i + 2], c[4 * i + 3], 0x0073), 0x5410);
}

// The same to nearest (ties to even).
template <bool SIGNED>
__device__ __forceinline__ void nearest_codes(const F2 (&x)[4], float inverse, Raw<1>& out) {
  uint32_t least = 0xFFu;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t half[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float lo, hi;
      f2_unpack(f2_mul(x[2 * i + j], f2_both(inverse)), lo, hi);
      uint16_t pair;
      asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(pair) : "f"(hi), "f"(lo));
      half[j] = pair;
      if (!SIGNED) least = min(least, min(half[j] & 0xFFu, half[j] >> 8));
    }
    out.w[i] = half[0] | (half[1] << 16);
  }
  if (!SIGNED && least == 0u) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float lo, hi;
      f2_unpack(x[i / 2], lo, hi);
      if (((out.w[i / 4] >> (8 * (i % 4))) & 0xFFu) == 0u && (i % 2 ? hi : lo) > 0.0f && inverse > 0.0f) out.w[i / 4] |= 1u << (8 * (i % 4));
    }
  }
}

// The largest magnitude of three, or a NaN if there is one.
__device__ __forceinline__ float largest3(float a, float b, float c) {
  float d;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// The largest magnitude of a block (a NaN, as a whole number, is above everything, and the scale becomes one), and what its elements are multiplied
// with for their codes: 448 times its reciprocal.
__device__ __forceinline__ float largest(const F2 (&x)[4], float& inverse) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) f2_unpack(x[i], f[2 * i], f[2 * i + 1]);
  const float mine = largest3(largest3(f[0], f[1], f[2]), largest3(f[3], f[4], f[5]), largest3(f[6], f[7], 0.0f));
  const float t = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(mine)));
  // 1 / t rounded, from the approximate reciprocal (of a quarter: it is normal for every t) and one correction on the remainder; times 448, rounded
  const float r = 0.25f * rcp_approx(0.25f * t);
  inverse = t >= kSmallest && t <= 3.4028235e38f ? kTopCode * fmaf(fmaf(-t, r, 1.0f), r, r) : 0.0f;
  return t;
}

template <bool SIGNED>
__device__ __forceinline__ void random_codes(const F2 (&x)[4], float top, float inverse, const uint4& bits, Raw<1>& out) {
  if (top <= 16384.0f) random_codes<SIGNED, false>(x, inverse * kTwoM120, bits, out);
  else random_codes<SIGNED, true>(x, inverse, bits, out);
}

// Everything of a lane's eight elements before the step, on its way from memory.
template <int PDT, int GDT, int BITS>
struct Loaded {
  Raw<Io<PDT>::kBytes> p;
  Raw<Io<GDT>::kBytes> g;
  Raw<BITS / 8> m, v;
  float ms, vs;
  template <bool QUAD, bool WHOLE>
  __device__ __forceinline__ void load(const StepTensor& t, const Spot<QUAD, WHOLE>& s, bool vec, uint64_t block) {
    g.load(t.g, s, vec);
    p.load(t.p, s, vec);
    m.load(t.m, s, vec);
    v.load(t.v, s, vec);
    if (BITS == 8) {
      ms = t.m_scale[block];
      vs = t.v_scale[block];
    }
  }
};

template <bool RANDOM, int PDT, int GDT, int BITS, bool QUAD, bool WHOLE>
__device__ __forceinline__ void step_block(const StepArgs& a, const StepTensor& t, const Rates& k, const SharedKey& key, uint64_t draw,
                                           const Loaded<PDT, GDT, BITS>& x, const Spot<QUAD, WHOLE>& s, bool vec, uint64_t block) {
  F2 p[4], g[4], m[4], r[4];
  x.g.get(g);
  x.p.get(p);
  x.m.get(m);
  x.v.get(r);
  if constexpr (BITS == 8) {
    moments(g, m, r, k, x.ms * (1.0f / kTopCode), x.vs * (1.0f / kTopCode));
  } else {  // v itself: v' = b2 v + (sqrt(1 - b2) g)^2
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m[i] = f2_fma(m[i], f2_both(a.beta1), f2_mul(g[i], f2_both(k.grad1)));
      const F2 b = f2_mul(g[i], f2_both(k.grad2));
      r[i] = f2_fma(b, b, f2_mul(r[i], f2_both(a.beta2)));
    }
    Raw<4> out;
    out.set(m);
    out.store(t.m, s, vec);
    out.set(r);
    out.store(t.v, s, vec);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float lo, hi;
      f2_unpack(r[i], lo, hi);
      r[i] = f2_pack(approx_sqrt(lo), approx_sqrt(hi));
    }
  }
  update(p, m, r, k.lr * t.decay * t.lr, k.first * t.lr, k.root, a.eps);
  if constexpr (PDT == kBF16 && RANDOM) {
    Raw<2> out;
    random_bf16(p, key.draw(draw | (1ull << 63), k.count), out);
    out.store(t.p, s, vec);
  } else {
    Raw<Io<PDT>::kBytes> out;
    out.set(p);
    out.store(t.p, s, vec);
  }
  if (PDT == kF32 && t.copy) {
    Raw<2> out;
    out.set(p);
    out.store(t.copy, s, vec);
  }
  if constexpr (BITS == 8) {
    float im, iv;
    if (!WHOLE && s.left < 8) {  // what does not exist has no part in the block's largest magnitude (m, v and g are zeros there, and so are these)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float lo, hi;
        f2_unpack(m[i], lo, hi);
        m[i] = f2_pack(2 * i < s.left ? lo : 0.0f, 2 * i + 1 < s.left ? hi : 0.0f);
        f2_unpack(r[i], lo, hi);
        r[i] = f2_pack(2 * i < s.left ? lo : 0.0f, 2 * i + 1 < s.left ? hi : 0.0f);
      }
    }
    const float top_m = largest(m, im), top_v = largest(r, iv);
    Raw<1> cm, cv;
    if constexpr (RANDOM) {
      const uint4 bits = key.draw(draw, k.count);
      random_codes<true>(m, top_m, im, bits, cm);
      random_codes<false>(r, top_v, iv, bits, cv);
    } else {
      nearest_codes<true>(m, im, cm);
      nearest_codes<false>(r, iv, cv);
    }
    cm.store(t.m, s, vec);
    cv.store(t.v, s, vec);
    if ((threadIdx.x & 31u) == 0) {
      t.m_scale[block] = top_m;
      t.v_scale[block] = top_v;
    }
  }
}

// CTAs of an SM (times here and below are of short runs, at the full clock, and those of 8-bit states of when the 302 M weights took 608 us, before
// `moments` rounded each operation; now five 684, four 698).  8-bit states: five, and two blocks of a warp's in registers at once (302 M weights, with four times as many CTAs as fit: 625 us;
// 645 with four an SM, 647 with six).  32-bit states: a block is 128 bytes a lane already, and six CTAs with one block each take 10.6 M weights at odd places
// in 49.6 us, four with two 56.
template <int BITS> constexpr int kStepCtas = BITS == 8 ? 5 : 6;

template <int PDT, int GDT, int BITS, bool RANDOM>
__global__ void __launch_bounds__(kStepThreads, kStepCtas<BITS>) adamw_kernel(const __grid_constant__ StepArgs a) {
  // random bits and 8-bit blocks are counted from the tensor's first element, and its vectors with them
  constexpr bool COUNTED = RANDOM || BITS == 8, QUAD = !COUNTED;
  __shared__ uint4 keys[5];
  enter_grid();
  const uint32_t lane = threadIdx.x & 31u;
  if constexpr (RANDOM) {
    if (threadIdx.x < 5) {
      const PhiloxKey key(a.rng[0]);
#pragma unroll
      for (int i = 0; i < 5; ++i)
        if (threadIdx.x == i) keys[i] = make_uint4(key.k0[2 * i], key.k1[2 * i], key.k0[2 * i + 1], key.k1[2 * i + 1]);
    }
    __syncthreads();
  }
  const SharedKey key{keys};
  float scale = a.control[2];
  Rates k;
  k.lr = a.control[0];
  if (a.clip) {
    const float norm = a.clip[0];
    if (!(fabsf(norm) <= 3.4028235e38f)) return;  // gradients that overflowed: nothing is changed
    scale *= a.clip[1];
  }
  const float number = a.control[1];
  k.first = __fdiv_rn(k.lr, -expm1f(number * a.log_beta1));
  k.root = __frsqrt_rn(-expm1f(number * a.log_beta2));
  k.grad1 = scale * a.one_beta1;
  k.grad2 = scale * a.root_one_beta2;
  k.scale = scale;
  k.one1 = a.one_beta1;
  k.one2 = a.one_beta2;
  k.beta2 = a.beta2;
  k.count = RANDOM ? a.rng[1] + a.site : 0ull;
  const uint32_t split = BITS == 8 ? a.split : 0u, blocks = a.chunk_blocks >> split;
  for (uint64_t part = (uint64_t)blockIdx.x * kStepWarps + (threadIdx.x >> 5); part < (uint64_t)a.n_chunks << split;
       part += (uint64_t)gridDim.x * kStepWarps) {
    const uint32_t c = (uint32_t)(part >> split);
    const StepTensor t = a.tensors[a.owner[c]];
    const uint64_t block = (part - ((uint64_t)t.chunk0 << split)) * blocks, from = block * kStepBlock;
    const bool vec = COUNTED ? t.head == 0u : t.head != kStepScalar;
    const uint32_t head = vec ? t.head : 0u;
    if (QUAD && head && from == 0) {  // the elements before the grid, as a block of two lanes'
      const uint64_t n = t.n < head ? t.n : head;
      const Spot<QUAD> s{4 * lane, (int32_t)(n > 4 * lane ? (n - 4 * lane < 4 ? n - 4 * lane : 4) : 0)};
      Loaded<PDT, GDT, BITS> x;
      x.load(t, s, false, 0);
      step_block<RANDOM>(a, t, k, key, 0, x, s, false, 0);
    }
    const uint64_t draw = (t.block0 + block) * 32 + lane;
    const uint64_t base = head + from + (QUAD ? 4 : 8) * lane;  // the lane's first element in block 0 of the chunk
    const uint64_t rest = t.n > head + from ? t.n - head - from : 0;  // of the tensor from this chunk on
    if (vec && blocks > 1 && rest >= (uint64_t)blocks * kStepBlock) {
      const auto spot = [&](uint32_t i) { return Spot<QUAD, true>{base + i * kStepBlock, 256}; };
      Loaded<PDT, GDT, BITS> x;
      if constexpr (BITS == 8) {  // the next block is on its way while one is in work
        Loaded<PDT, GDT, BITS> y;
        x.load(t, spot(0), true, block);
#pragma unroll 1
        for (uint32_t i = 0; i < blocks; i += 2) {
          y.load(t, spot(i + 1), true, block + i + 1);
          step_block<RANDOM>(a, t, k, key, draw + 32 * i, x, spot(i), true, block + i);
          if (i + 2 < blocks) x.load(t, spot(i + 2), true, block + i + 2);
          step_block<RANDOM>(a, t, k, key, draw + 32 * (i + 1), y, spot(i + 1), true, block + i + 1);
        }
      } else {
#pragma unroll 1
        for (uint32_t i = 0; i < blocks; ++i) {
          x.load(t, spot(i), true, block + i);
          step_block<RANDOM>(a, t, k, key, draw + 32 * i, x, spot(i), true, block + i);
        }
      }
      continue;
    }
#pragma unroll 1
    for (uint32_t i = 0; i < blocks && (uint64_t)i * kStepBlock < rest; ++i) {
      const uint64_t first = base + i * kStepBlock;
      const Spot<QUAD> s{first, first >= t.n ? 0 : (t.n - first < 256 ? (int32_t)(t.n - first) : 256)};
      Loaded<PDT, GDT, BITS> x;
      x.load(t, s, vec, block + i);
      step_block<RANDOM>(a, t, k, key, draw + 32 * i, x, s, vec, block + i);
    }
  }
}

// ---------------------------------------------------------------- the gradients' norm
// The sum of eight squares: in 32 bits where it comes out far from both ends of their range (no square overflowed, and none that vanished
// matters beside 2^-80), else in 64.
template <int GDT>
__device__ __forceinline__ float square_sum(const Raw<Io<GDT>::kBytes>& raw, double& wide) {
  F2 g[4];
  raw.get(g);
  float x, y;
  f2_unpack(f2_add(f2_fma(g[0], g[0], f2_mul(g[1], g[1])), f2_fma(g[2], g[2], f2_mul(g[3], g[3]))), x, y);
  const float s = x + y;
  if (s >= 8.271806e-25f && s <= 1.2676506e30f) return s;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f2_unpack(g[i], x, y);
    wide = fma((double)x, (double)x, fma((double)y, (double)y, wide));
  }
  return 0.0f;
}

constexpr uint32_t kAhead = 4;  // blocks in flight

// A warp's part of the squares: chunk `first` and those `stride` apart.  Eight chunks are looked up at once, by a lane each (2.9 M gradients
// 4.3 us; one chunk after another, each a chain of three reads, 8.1).
constexpr uint32_t kLooks = 8;

// SINGLE: chunks are single blocks.
template <int GDT, bool SINGLE>
__device__ __forceinline__ double chunk_squares(const StepArgs& a, uint32_t first, uint32_t stride) {
  constexpr int ES = Io<GDT>::kBytes;
  constexpr bool QUAD = ES == 4;
  const uint32_t lane = threadIdx.x & 31u;
  const int32_t place = (QUAD ? 4 : 8) * lane, chunk = (SINGLE ? 1 : a.chunk_blocks) * kStepBlock;
  double sum = 0.0;
  for (uint32_t base = first; base < a.n_chunks; base += kLooks * stride) {  // (chunks are fewer than 2^31)
    const uint32_t c = base + lane * stride;
    const bool mine = lane < kLooks && c < a.n_chunks;
    uint64_t at = 0;
    int32_t left = 0, head = 0, before = 0;  // elements of the chunk, before the grid, and of these in the tensor
    bool vec = false;
    if (mine) {
      const StepTensor& t = a.tensors[a.owner[c]];
      vec = t.head != kStepScalar;
      head = vec ? t.head : 0;
      const uint64_t from = head + (uint64_t)(c - t.chunk0) * chunk;
      at = (uint64_t)t.g + from * ES;
      left = from >= t.n ? 0 : (t.n - from < (uint64_t)chunk ? (int32_t)(t.n - from) : chunk);
      if (c == t.chunk0) before = t.n < (uint64_t)head ? (int32_t)t.n : head;
    }
    const int chunks = __popc(__ballot_sync(0xffffffffu, mine));
    const auto add = [&](const Raw<ES> (&raw)[kAhead]) {
      float s = 0.0f;
#pragma unroll
      for (uint32_t i = 0; i < kAhead; ++i) s += square_sum<GDT>(raw[i], sum);
      sum += (double)s;  // of 32 elements, each eight from 2^-80 to 2^100
    };
    if constexpr (SINGLE) {  // blocks of several chunks in flight
#pragma unroll 1
      for (int k = 0; k < chunks; k += kAhead) {
        Raw<ES> raw[kAhead];
#pragma unroll
        for (int i = 0; i < (int)kAhead; ++i) {
          const int32_t n = __shfl_sync(0xffffffffu, left, k + i) - place;
          const uint64_t from = __shfl_sync(0xffffffffu, at, k + i);
          const bool wide = __shfl_sync(0xffffffffu, (int)vec, k + i) != 0;
          raw[i].load((const void*)from, Spot<QUAD>{(uint64_t)place, n < 0 ? 0 : n}, wide);
        }
        add(raw);
      }
    } else {
#pragma unroll 1
      for (int k = 0; k < chunks; ++k) {
        int32_t n = __shfl_sync(0xffffffffu, left, k);
        uint64_t from = __shfl_sync(0xffffffffu, at, k);
        const bool wide = __shfl_sync(0xffffffffu, (int)vec, k) != 0;
#pragma unroll 1
        for (; n > 0; n -= kAhead * kStepBlock, from += kAhead * kStepBlock * ES) {
          Raw<ES> raw[kAhead];
          if (wide && n >= (int32_t)(kAhead * kStepBlock)) {
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) raw[i].load((const void*)from, Spot<QUAD, true>{place + i * kStepBlock, 256}, true);
          } else {
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) {
              const int32_t rest = n - (int32_t)(i * kStepBlock) - place;
              raw[i].load((const void*)from, Spot<QUAD>{place + i * kStepBlock, rest < 0 ? 0 : (rest < 256 ? rest : 256)}, wide);
            }
          }
          add(raw);
        }
      }
    }
    for (uint32_t rest = __ballot_sync(0xffffffffu, before > 0); rest; rest &= rest - 1) {  // the elements before the grid, at most seven
      const int i = __ffs(rest) - 1;
      const int32_t n = __shfl_sync(0xffffffffu, before, i) - (int32_t)(4 * lane);
      const uint64_t from = __shfl_sync(0xffffffffu, at, i) - (uint64_t)__shfl_sync(0xffffffffu, head, i) * ES;
      Raw<ES> front;
      front.load((const void*)from, Spot<true>{4 * lane, n < 0 ? 0 : (n < 4 ? n : 4)}, false);
      const float s = square_sum<GDT>(front, sum);
      sum += (double)s;
    }
  }
  return sum;
}

template <int GDT, bool SINGLE>
__global__ void __launch_bounds__(kNormThreads, 4) grad_norm_kernel(const __grid_constant__ StepArgs a, double* partials) {
  __shared__ double buf[kNormWarps];
  enter_grid();
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  double sum = chunk_squares<GDT, SINGLE>(a, blockIdx.x * kNormWarps + warp, gridDim.x * kNormWarps);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) buf[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kNormWarps; ++w) sum += buf[w];
    partials[blockIdx.x] = sum;
  }
}

__device__ __forceinline__ void write_norm(double sum, float scale, float max_norm, float* out) {
  const double norm = sqrt(sum) * fabs((double)scale);
  const double factor = (double)max_norm / (norm + 1e-6);
  out[0] = (float)norm;
  out[1] = (float)(factor > 1.0 ? 1.0 : factor);
}

constexpr int kFinishThreads = 256;

__global__ void __launch_bounds__(kFinishThreads) grad_norm_finish_kernel(const double* partials, uint32_t n, const float* control, float max_norm,
                                                                float* out) {
  __shared__ double buf[kFinishThreads / 32];
  enter_grid();
  const float scale = control[2];
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < (kMaxNormCtas + kFinishThreads - 1) / kFinishThreads; ++i) {
    const uint32_t at = threadIdx.x + i * kFinishThreads;
    if (at < n) sum += partials[at];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (threadIdx.x % 32 == 0) buf[threadIdx.x / 32] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kFinishThreads / 32; ++w) sum += buf[w];
    write_norm(sum, scale, max_norm, out);
  }
}

// Plans of few chunks, of one block each: one cluster, whose CTAs leave their sums in the first one's shared memory, in the place of a second
// launch.  Up to 2048 chunks are faster so (16 384 gradients 2.6 us, two kernels
// 3.1; 0.5 M 3.4, 3.9), and the host saves a launch; at 4090 both take 4.4 us.  Clusters of eight, the portable size, take 4.3 us for 0.5 M.
constexpr int kFewCtas = 16, kFewWarps = 16;

template <int GDT>
__global__ void __cluster_dims__(kFewCtas) __launch_bounds__(kFewWarps * 32)
    grad_norm_few_kernel(const __grid_constant__ StepArgs a, float max_norm, float* out) {
  __shared__ double buf[kFewWarps], all[kFewCtas];
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");  // "this CTA has started": awaited before one writes to another
  enter_grid();
  const float scale = a.control[2];
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  double sum = chunk_squares<GDT, true>(a, warp * kFewCtas + blockIdx.x, kFewCtas * kFewWarps);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) buf[warp] = sum;
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kFewWarps; ++w) sum += buf[w];
    uint32_t there;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(there) : "r"((uint32_t)__cvta_generic_to_shared(&all[blockIdx.x])));
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(there), "d"(sum) : "memory");
  }
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (blockIdx.x == 0 && threadIdx.x < 32) {
    sum = threadIdx.x < kFewCtas ? all[threadIdx.x] : 0.0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (threadIdx.x == 0) write_norm(sum, scale, max_norm, out);
  }
}

// Whether the current device has room for a cluster of sixteen: a part of a GPU, or one with SMs switched off, may not.  Asked once a device.
template <int GDT>
bool few_fits() {
  static std::atomic<uint64_t> asked{0}, fits{0};  // a bit for each device
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev < 64 && (asked.load(std::memory_order_acquire) & bit)) return (fits.load(std::memory_order_relaxed) & bit) != 0;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kFewCtas;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kFewCtas);
  cfg.blockDim = dim3(kFewWarps * 32);
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  const bool ok = cudaFuncSetAttribute(grad_norm_few_kernel<GDT>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                  cudaOccupancyMaxActiveClusters(&n, grad_norm_few_kernel<GDT>, &cfg) == cudaSuccess && n > 0;
  if (!ok) cudaGetLastError();  // the other kernels run: nobody is to find this error later
  if (dev < 64) {
    if (ok) fits.fetch_or(bit, std::memory_order_relaxed);
    asked.fetch_or(bit, std::memory_order_release);
  }
  return ok;
}

template <int PDT, int GDT>
cudaError_t launch_adamw_types(int bits, const StepArgs& a, unsigned grid, cudaStream_t st) {
  if (bits == 32) {
    if constexpr (PDT == kBF16)  // binary32 weights and states need no rounding
      if (a.rng) return launch_overlapped(adamw_kernel<PDT, GDT, 32, true>, dim3(grid), kStepThreads, 0, st, a);
    return launch_overlapped(adamw_kernel<PDT, GDT, 32, false>, dim3(grid), kStepThreads, 0, st, a);
  }
  return a.rng ? launch_overlapped(adamw_kernel<PDT, GDT, 8, true>, dim3(grid), kStepThreads, 0, st, a)
               : launch_overlapped(adamw_kernel<PDT, GDT, 8, false>, dim3(grid), kStepThreads, 0, st, a);
}

}  // namespace

cudaError_t launch_adamw(int pdt, int gdt, int state_bits, StepArgs a, cudaStream_t st) {
  if (a.n_chunks == 0) return cudaSuccess;
  // 8-bit states: chunks of four blocks in halves, the two blocks that are in registers at once (8.0 M weights 24 us, whole 27.5; 28 M 71 and 77);
  // chunks of sixteen whole (302 M weights 608 us, 698 in parts of two to eight)
  a.split = state_bits == 8 && a.chunk_blocks == 4 ? 1 : 0;
  const uint64_t resident = (uint64_t)sm_count() * (state_bits == 8 ? kStepCtas<8> : kStepCtas<32>);  // CTAs at once
  // Sixteen times as many CTAs as fit, whose last ones even out what the SMs have left (302 M weights: 32-bit states 1298 us, 1397 with as many as
  // fit; 8-bit states 608, 650); where 8-bit states have few blocks a CTA, its start counts for more (2.4 M weights 10.5 us, 13.6 with four times
  // as many as fit).
  const uint64_t want = (((uint64_t)a.n_chunks << a.split) + kStepWarps - 1) / kStepWarps, cap = resident * (state_bits == 8 && a.chunk_blocks < 16 ? 1 : 16);
  const unsigned grid = (unsigned)(want < cap ? want : cap);
  if (pdt == kF32)
    return gdt == kF32 ? launch_adamw_types<kF32, kF32>(state_bits, a, grid, st) : launch_adamw_types<kF32, kBF16>(state_bits, a, grid, st);
  return gdt == kF32 ? launch_adamw_types<kBF16, kF32>(state_bits, a, grid, st) : launch_adamw_types<kBF16, kBF16>(state_bits, a, grid, st);
}

// As many CTAs as fit a B200 at most, whatever the device: the scratch is sized by them.
uint64_t grad_norm_scratch_bytes(uint32_t n_chunks) {
  const uint64_t want = ((uint64_t)n_chunks + kNormWarps - 1) / kNormWarps;
  return (want < 1 ? 1 : (want < kMaxNormCtas ? want : kMaxNormCtas)) * sizeof(double);
}

cudaError_t launch_grad_norm(int gdt, const StepArgs& a, float max_norm, float* out, double* scratch, cudaStream_t st) {
  if (a.chunk_blocks == 1 && a.n_chunks <= kFewCtas * kFewWarps * kLooks && (gdt == kF32 ? few_fits<kF32>() : few_fits<kBF16>()))
    return launch_overlapped(gdt == kF32 ? grad_norm_few_kernel<kF32> : grad_norm_few_kernel<kBF16>, dim3(kFewCtas), kFewWarps * 32, 0, st, a, max_norm, out);
  const unsigned grid = (unsigned)(grad_norm_scratch_bytes(a.n_chunks) / sizeof(double));
  const auto go = [&](void (*kernel)(const StepArgs, double*)) { return launch_overlapped(kernel, dim3(grid), kNormThreads, 0, st, a, scratch); };
  const cudaError_t e = a.chunk_blocks == 1 ? (gdt == kF32 ? go(grad_norm_kernel<kF32, true>) : go(grad_norm_kernel<kBF16, true>))
                                            : (gdt == kF32 ? go(grad_norm_kernel<kF32, false>) : go(grad_norm_kernel<kBF16, false>));
  if (e != cudaSuccess) return e;
  return launch_overlapped(grad_norm_finish_kernel, dim3(1), kFinishThreads, 0, st, (const double*)scratch, grid, a.control, max_norm, out);
}

}  // namespace s2a
