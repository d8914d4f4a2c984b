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
// as K slots of two vectors of V; in the layout of halves a turning slot's vectors are rot / 2 elements apart, so that pairs never cross
// lanes.  A warp takes 32 / L rows (L lanes a row) at a time: a group.  Where a token has as many rows (heads of queries and keys) or more,
// its groups follow one another and its cosines and sines are computed once; where it has fewer, a group takes the rows of several tokens.  The
// phases are computed by all lanes, each some pairs, and shared through the warp's own shared memory.  Rows come through a ring of
// asynchronous copies of each warp's own, four groups deep (the norm's backward: kBwdStages).  With plain loads, addresses from scratch and the weights read per token, the norm
// of [64, 197, 12 + 12, 64] bfloat16 took 581 instructions a group and 39.5 us; so it takes 17.0 (a copy of the same bytes: 13.5), the rotation of
// [2, 16384, 32 + 8, 128] 121 to 123 us (0.84 of a copy's rate) and the norm's backward of [4, 4097, 32 + 8, 128] 92 (0.83), or 100 to 102 (0.76) in runs of a
// second, at the 1.77 GHz that the power limit leaves.
//
// Rows that turn as a whole and are 2, 4, 6, 8, 10, 12 or 16 lanes (heads of 32 to 256, whose halves are whole 32-byte sectors) have kernels of their
// own (L > 0), in which every slot exists and each lane copies for itself; the others (L = 0) ask for each slot and copy by vectors of W elements in order.
#pragma once

#include <algorithm>

#include "s2a_launch.h"
#include "s2a_oct.cuh"

namespace s2a {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kLaneElems = 16;
// Stages of a warp's ring: groups of rows in flight or in work.  Two tensors have five in bfloat16 ([4, 4097, 32 + 8, 128]
// backward 94 us, 100 with four) and three in binary32, so that two CTAs fit an SM.
template <int DT> constexpr int kBwdStages = DT == kF32 ? 3 : 5;

// Where a warp's lanes stand in a group of rows: `row` of the group, and what that is: row `head` (plus groups already done) of token `token`
// of the group's.
template <int L, bool MULTI>
struct Lane {
  uint32_t slot, row, head, token, per;  // slot of k = 0; per: rows of a token that a group takes
  bool on;
  __device__ __forceinline__ Lane(const RopeArgs& a, uint32_t heads, uint32_t group_tokens) {
    const uint32_t lane = threadIdx.x & 31u, n = lanes(a), rows = L ? 32 / (L ? L : 1) : a.rows_per_warp;
    row = lane / n;
    slot = lane - row * n;
    on = row < rows;  // (always, where L divides 32)
    if (MULTI && group_tokens > 1) {  // all rows of several tokens
      token = row / heads;
      head = row - token * heads;
      per = heads;
      on = on && token < group_tokens;
    } else {
      token = 0;
      head = row;
      per = rows;
    }
  }
  static __device__ __forceinline__ uint32_t lanes(const RopeArgs& a) { return L ? L : a.lanes; }
  __device__ __forceinline__ bool leads() const { return on && slot == 0 && head == 0; }  // a token's first lane
};

// (cos, sin) of turn * pos, times `scale`; `sign` turns back.  The fraction's top 32 bits: a quarter turn to the nearest, and what
// is left of it, at most an eighth of a turn, for which Taylor's polynomials to x^9 and x^10 are off by 2e-9 and 1e-10.
__device__ __forceinline__ float2 phase(uint64_t turn, int64_t pos, float scale, float sign) {
  const uint32_t top = (uint32_t)((turn * (uint64_t)pos) >> 32);
  const uint32_t quarter = (top + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(top - (quarter << 30)) * 1.4629180792671596e-09f;  // radians: 2 pi / 2^32
  const float z = x * x;
  float s = fmaf(z, fmaf(z, fmaf(z, fmaf(z, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f) * x, x);
  float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.0f);
  // a quarter more: (c, s) becomes (-s, c); a half more: both signs
  const float u = (quarter & 1u) ? -s : c, v = (quarter & 1u) ? c : s;
  const float turned = (quarter & 2u) ? -scale : scale;
  return make_float2(u * turned, v * (turned * sign));
}

template <int BYTES> struct RawOf;
template <> struct RawOf<16> { using T = uint4; };
template <> struct RawOf<8> { using T = uint2; };
template <> struct RawOf<4> { using T = uint32_t; };
template <> struct RawOf<2> { using T = uint16_t; };

// A vector of V elements as F2s: V / 2, or one with nothing in its upper half.
template <int V> constexpr int kHalf = V > 1 ? V / 2 : 1;

template <int DT, int V>
__device__ __forceinline__ void read_vector(const void* p, F2 (&f)[kHalf<V>]) {
  if constexpr (DT == kF32) {
    if constexpr (V == 4) {
      const ulonglong2 r = *(const ulonglong2*)p;
      f[0].v = r.x;
      f[1].v = r.y;
    } else if constexpr (V == 2) {
      f[0].v = *(const unsigned long long*)p;
    } else {
      f[0] = f2_pack(*(const float*)p, 0.0f);
    }
  } else if constexpr (V == 8) {
    const uint4 r = *(const uint4*)p;
    f[0] = f2_from_bf16x2(r.x);
    f[1] = f2_from_bf16x2(r.y);
    f[2] = f2_from_bf16x2(r.z);
    f[3] = f2_from_bf16x2(r.w);
  } else if constexpr (V == 4) {
    const uint2 r = *(const uint2*)p;
    f[0] = f2_from_bf16x2(r.x);
    f[1] = f2_from_bf16x2(r.y);
  } else if constexpr (V == 2) {
    f[0] = f2_from_bf16x2(*(const uint32_t*)p);
  } else {
    f[0] = f2_pack(__uint_as_float((uint32_t) * (const uint16_t*)p << 16), 0.0f);
  }
}

template <int DT, int V>
__device__ __forceinline__ void write_vector(void* p, const F2 (&f)[kHalf<V>]) {
  if constexpr (DT == kF32) {
    if constexpr (V == 4) {
      *(ulonglong2*)p = make_ulonglong2(f[0].v, f[1].v);
    } else if constexpr (V == 2) {
      *(unsigned long long*)p = f[0].v;
    } else {
      float a, b;
      f2_unpack(f[0], a, b);
      *(float*)p = a;
    }
  } else if constexpr (V == 8) {
    *(uint4*)p = make_uint4(f2_to_bf16x2(f[0]), f2_to_bf16x2(f[1]), f2_to_bf16x2(f[2]), f2_to_bf16x2(f[3]));
  } else if constexpr (V == 4) {
    *(uint2*)p = make_uint2(f2_to_bf16x2(f[0]), f2_to_bf16x2(f[1]));
  } else if constexpr (V == 2) {
    *(uint32_t*)p = f2_to_bf16x2(f[0]);
  } else {
    float a, b;
    f2_unpack(f[0], a, b);
    *(__nv_bfloat16*)p = __float2bfloat16_rn(a);
  }
}

// V binary32 numbers of shared memory, on a boundary of V of them (16 bytes at most).
template <int V>
__device__ __forceinline__ void read_floats(const float* p, F2 (&f)[kHalf<V>]) {
  if constexpr (V >= 4) {
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
      const ulonglong2 r = ((const ulonglong2*)p)[i];
      f[2 * i].v = r.x;
      f[2 * i + 1].v = r.y;
    }
  } else if constexpr (V == 2) {
    f[0].v = *(const unsigned long long*)p;
  } else {
    f[0] = f2_pack(*p, 0.0f);
  }
}

// A lane's places in a row, the same in every row of a launch: the two vectors of each slot, which of them exist, and which turn.  Halves: a
// slot that turns holds V pairs (both vectors turn), the others two neighbouring vectors.  Interleaved (pairs lie within vectors): vectors s and
// s + slots, each with V / 2 pairs of its own.
template <int V, int K, bool INTER, int L, bool MULTI>
struct Places {
  uint32_t at[K], to[K];  // elements of the first and the second vector
  uint32_t pair[K], pair2[K];  // first pair of the first and, interleaved, of the second vector
  uint32_t first, second, turns, turns2;  // bits
  __device__ __forceinline__ bool has_first(int k) const { return L || ((first >> k) & 1u); }
  __device__ __forceinline__ bool has_second(int k) const { return L || ((second >> k) & 1u); }
  __device__ __forceinline__ bool turning(int k) const { return L || ((turns >> k) & 1u); }
  __device__ __forceinline__ bool turning2(int k) const { return L || ((turns2 >> k) & 1u); }
  __device__ __forceinline__ Places(const RopeArgs& a, const Lane<L, MULTI>& l) {
    first = second = turns = turns2 = 0u;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t s = l.slot + k * Lane<L, MULTI>::lanes(a);
      const uint32_t pairs = L ? L * kLaneElems / 2 : a.pairs;
      at[k] = to[k] = pair[k] = pair2[k] = 0u;
      if (!L && (!l.on || s >= a.slots)) continue;
      first |= 1u << k;
      if (INTER && !L) {
        at[k] = V * s;
        to[k] = V * (s + a.slots);
        if (to[k] < a.head_dim) second |= 1u << k;
        else to[k] = at[k];
        if (at[k] < 2 * pairs) {
          turns |= 1u << k;
          pair[k] = at[k] / 2;
        }
        if (((second >> k) & 1u) && to[k] < 2 * pairs) {
          turns2 |= 1u << k;
          pair2[k] = to[k] / 2;
        }
      } else if (L || s < a.turn_slots) {
        turns |= 1u << k;
        turns2 |= 1u << k;
        second |= 1u << k;
        if (V == 1) {  // single pairs: adjacent, or half apart
          at[k] = a.interleaved ? 2 * s : s;
          to[k] = a.interleaved ? 2 * s + 1 : s + pairs;
          pair[k] = s;
        } else {
          at[k] = V * s;
          to[k] = V * s + pairs;
          pair[k] = INTER ? at[k] / 2 : at[k];
          pair2[k] = INTER ? to[k] / 2 : 0u;
        }
      } else {
        at[k] = 2 * pairs + 2 * V * (s - a.turn_slots);
        to[k] = at[k] + V;
        if (to[k] < a.head_dim) second |= 1u << k;
        else to[k] = at[k];
      }
    }
  }
};

// A lane's cosines and sines, of the slots that turn.
template <int V, int K, bool INTER, int L, bool MULTI>
struct Angles {
  F2 c[K][kHalf<V>], s[K][kHalf<V>];  // of the pairs in order
  __device__ __forceinline__ void read(const Places<V, K, INTER, L, MULTI>& p, const float* cs, const float* sn) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if constexpr (INTER) {  // what does not turn reads the first pairs, and is not turned
        read_part(cs + p.pair[k], cs + p.pair2[k], c[k]);
        read_part(sn + p.pair[k], sn + p.pair2[k], s[k]);
      } else {
        if (!p.turning(k)) continue;
        read_floats<V>(cs + p.pair[k], c[k]);
        read_floats<V>(sn + p.pair[k], s[k]);
      }
    }
  }
  // V / 2 numbers from each of two places
  static __device__ __forceinline__ void read_part(const float* p, const float* q, F2 (&f)[kHalf<V>]) {
    if constexpr (V == 2) {
      f[0] = f2_pack(*p, *q);
    } else {
      F2 x[kHalf<V / 2>], y[kHalf<V / 2>];
      read_floats<V / 2>(p, x);
      read_floats<V / 2>(q, y);
#pragma unroll
      for (int i = 0; i < V / 4; ++i) {
        f[i] = x[i];
        f[V / 4 + i] = y[i];
      }
    }
  }
  static __device__ __forceinline__ F2 turn_pair(F2 x, float c, float s) {
    float a, b;
    f2_unpack(x, a, b);
    return f2_pack(fmaf(a, c, -(b * s)), fmaf(a, s, b * c));
  }
  __device__ __forceinline__ void turn(const Places<V, K, INTER, L, MULTI>& p, int k, F2 (&a)[kHalf<V>], F2 (&b)[kHalf<V>]) const {
    if constexpr (INTER) {
      if (p.turning(k)) {
#pragma unroll
        for (int j = 0; j < V / 2; ++j) turn_one(a[j], c[k], s[k], j);
      }
      if (p.turning2(k)) {
#pragma unroll
        for (int j = 0; j < V / 2; ++j) turn_one(b[j], c[k], s[k], V / 2 + j);
      }
    } else if (p.turning(k)) {  // two pairs an instruction
#pragma unroll
      for (int j = 0; j < kHalf<V>; ++j) {
        const F2 u = f2_sub(f2_mul(a[j], c[k][j]), f2_mul(b[j], s[k][j]));
        b[j] = f2_fma(a[j], s[k][j], f2_mul(b[j], c[k][j]));
        a[j] = u;
      }
    }
  }
  static __device__ __forceinline__ void turn_one(F2& x, const F2 (&cc)[kHalf<V>], const F2 (&ss)[kHalf<V>], int i) {
    float c0, c1, s0, s1;
    f2_unpack(cc[i / 2], c0, c1);
    f2_unpack(ss[i / 2], s0, s1);
    x = turn_pair(x, i % 2 ? c1 : c0, i % 2 ? s1 : s0);
  }
};

// A warp's part of all groups of rows: an even share of neighbouring ones.  The tokens are counted through the sequences first, so that
// neighbours have the same place in their sequences and, as a rule, the same position, whose cosines then stay.  Where a group takes several
// tokens, each lane walks along its own.
template <bool MULTI>
struct Walk {
  uint32_t b, t, i, left;  // sequence and token of the lane, group of rows of the token, groups left
  __device__ __forceinline__ Walk(const RopeArgs& a, uint32_t warp, int which, uint32_t groups, uint32_t token) {
    // the first `more` warps have one more
    const uint32_t share = a.share[which], more = a.more[which], start = warp * share + (warp < more ? warp : more);
    left = share + (warp < more ? 1u : 0u);
    uint32_t n = start / groups;
    i = start - n * groups;
    if (MULTI) n = n * a.group_tokens[which] + token;
    t = n / a.batch;
    b = n - t * a.batch;
  }
  // true where new tokens begin
  __device__ __forceinline__ bool next(const RopeArgs& a, int which, uint32_t groups) {
    --left;
    if (++i < groups) return false;
    i = 0;
    if (!MULTI) {
      if (++b < a.batch) return true;
      b = 0;
    } else {
      b += a.step_b[which];
      t += a.step_t[which];
      if (b < a.batch) return true;
      b -= a.batch;
    }
    ++t;
    return true;
  }
  // the same for one that only counts
  __device__ __forceinline__ bool count(uint32_t groups) {
    --left;
    if (++i < groups) return false;
    i = 0;
    return true;
  }
  __device__ __forceinline__ bool there(const RopeArgs& a) const { return !MULTI || t < a.tokens; }
  __device__ __forceinline__ uint64_t row0(const HeadsArg& h) const { return (uint64_t)h.data + b * h.batch + t * h.token; }
};

// A copy of BYTES at constant offsets from both addresses, or zeros where there is nothing.
template <int BYTES, int TO, int FROM>
__device__ __forceinline__ void copy_or_zero(uint32_t to, uint64_t from, bool there) {
  if constexpr (BYTES == 16)
    asm volatile("cp.async.cg.shared.global [%0+%3], [%1+%4], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0), "n"(TO), "n"(FROM) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0+%4], [%1+%5], %2, %3;" ::"r"(to), "l"(from), "n"(BYTES), "r"(there ? BYTES : 0), "n"(TO), "n"(FROM)
                 : "memory");
}

// A warp's group of rows in a stage of its ring.  Rows with kernels of their own (L > 0): each lane copies what it will read, to a place
// of its own, and writes from registers.  Others: their rows lie one behind the other, copied by vectors of W in order, so that neighbouring lanes
// have neighbouring vectors whatever the row's length, read by each lane at its places, and written back the same way ([3, 16 + 16, 2001,
// 80] binary32, half turning: 36.9 us with each lane's own copies, most of which cut 32-byte sectors).  Behind the rows of a stage stand 16
// bytes of zeros, which a lane reads in the place of a vector that does not exist.
template <int DT, int V, int W, int K, int L, bool MULTI>
struct Group {
  static constexpr int kBytes = W * Io<DT>::kBytes;
  static constexpr int kCopies = kLaneElems / W;  // vectors of a lane
  static constexpr int kRowsBytes = kCopies * 32 * kBytes;
  static constexpr int kGroupBytes = kRowsBytes + (L ? 0 : 16);  // of a warp
  static constexpr int kApart = L * (kLaneElems / 2) * Io<DT>::kBytes;  // bytes from the first half of a row to the second
  static constexpr bool kKept = kCopies <= 4;
  uint32_t vectors, inverse;                    // L = 0: vectors of a row, and 2^20 / that, rounded up: j / vectors is exact for j < 512
  uint32_t lane_of[kKept ? kCopies : 1], byte_of[kKept ? kCopies : 1];  // of the lane's vectors, where they are few: a lane of the row, and the place in it
  uint32_t off_a[L ? 1 : K], off_b[L ? 1 : K];  // where the lane's two vectors of a slot lie in a stage
  template <typename P>
  __device__ __forceinline__ Group(const RopeArgs& a, const Lane<L, MULTI>& l, const P& p) {
    if constexpr (L == 0) {
      vectors = a.head_dim / W;
      inverse = (1048576u + vectors - 1) / vectors;
      if constexpr (kKept)
#pragma unroll
        for (int m = 0; m < kCopies; ++m) split(m, a, lane_of[m], byte_of[m]);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const uint32_t row = l.row * vectors * kBytes;
        off_a[k] = p.has_first(k) ? row + p.at[k] * Io<DT>::kBytes : kRowsBytes;
        off_b[k] = p.has_second(k) ? row + p.to[k] * Io<DT>::kBytes : kRowsBytes;
      }
    }
  }
  // MULTI: a lane of the vector's row, 32 behind the last row; else the row itself, far beyond any behind the last
  __device__ __forceinline__ void split(int m, const RopeArgs& a, uint32_t& lane, uint32_t& byte) const {
    const uint32_t j = m * 32 + (threadIdx.x & 31u), r = (j * inverse) >> 20;
    byte = (j - r * vectors) * kBytes;
    if (MULTI) lane = r < a.rows_per_warp ? r * a.lanes : 32u;
    else lane = r < a.rows_per_warp ? r : 0x40000000u;
  }
  // The address of the lane's m-th vector; 0 where there is none.  MULTI: given each lane's row (0: none), as the rows belong to several tokens; else
  // given the group's first row.
  template <typename S>
  __device__ __forceinline__ uint64_t vector(int m, const RopeArgs& a, uint64_t row, const S& rows, uint32_t first) const {
    uint32_t lane, byte;
    if constexpr (kKept) {
      lane = lane_of[m];
      byte = byte_of[m];
    } else {
      split(m, a, lane, byte);
    }
    if constexpr (MULTI) {
      const uint64_t from = __shfl_sync(0xffffffffu, row, lane & 31u);
      return lane < 32u && from ? from + byte : 0;
    } else {
      return first + lane < rows.heads ? rows.row(first + lane) + byte : 0;
    }
  }
  __device__ __forceinline__ void clear(char* ring, uint32_t groups) const {
    if (L == 0 && (threadIdx.x & 31u) < groups) *(uint4*)(ring + (threadIdx.x & 31u) * kGroupBytes + kRowsBytes) = make_uint4(0u, 0u, 0u, 0u);
  }

  // Rows of a token: row r of the queries lies at q + r * q_head vectors; with KEYS those from heads0 on are the keys', at k + r * k_head vectors.
  template <bool KEYS>
  struct Source {
    uint64_t q, k;
    uint32_t q_head, k_head, heads0, heads;
    __device__ __forceinline__ Source(const HeadsArg& hq, const HeadsArg& hk, uint32_t h0, uint32_t h)
        : q(0), k(0), q_head((uint32_t)(hq.head / kBytes)), k_head((uint32_t)(hk.head / kBytes)), heads0(h0), heads(h) {}
    __device__ __forceinline__ uint64_t row(uint32_t r) const {
      if (!KEYS) return q + (uint64_t)(r * kBytes) * q_head;
      const bool keys = r >= heads0;
      return (keys ? k : q) + (uint64_t)(r * kBytes) * (keys ? k_head : q_head);
    }
    // on to the walk's token
    __device__ __forceinline__ void enter(const Walk<MULTI>& w, const HeadsArg& hq, const HeadsArg& hk) {
      q = w.row0(hq);
      if (KEYS) k = w.row0(hk) - heads0 * hk.head;
    }
  };

  // first: the group's first row of the token; r: the lane's; there: whether it exists
  template <typename S>
  __device__ __forceinline__ void fetch(char* stage, const RopeArgs& a, const S& from, uint32_t first, uint32_t r, bool there,
                                        const Lane<L, MULTI>& l) const {
    const uint32_t lane = threadIdx.x & 31u;
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(stage) + lane * kBytes;
    if constexpr (L > 0) {
      const uint64_t row = from.row(r) + l.slot * kBytes;
      copy_or_zero<kBytes, 0, 0>(to, row, there);
      copy_or_zero<kBytes, 32 * kBytes, kApart>(to, row, there);
      if constexpr (K == 2) {
        copy_or_zero<kBytes, 64 * kBytes, L * kBytes>(to, row, there);
        copy_or_zero<kBytes, 96 * kBytes, L * kBytes + kApart>(to, row, there);
      }
    } else {
      const uint64_t row = MULTI && there ? from.row(r) : 0;
#pragma unroll
      for (int m = 0; m < kCopies; ++m) {
        const uint64_t at = vector(m, a, row, from, first);
        if constexpr (kBytes >= 4) copy_or_zero<kBytes, 0, 0>(to + m * 32 * kBytes, at, at != 0);
        else *(uint16_t*)(stage + (m * 32 + lane) * kBytes) = at ? *(const uint16_t*)at : (uint16_t)0;
      }
    }
  }
  __device__ __forceinline__ void read(const char* stage, int k, F2 (&a)[kHalf<V>], F2 (&b)[kHalf<V>]) const {
    if constexpr (L > 0) {
      const char* own = stage + (2 * k * 32 + (threadIdx.x & 31u)) * kBytes;
      read_vector<DT, V>(own, a);
      read_vector<DT, V>(own + 32 * kBytes, b);
    } else {
      read_vector<DT, V>(stage + off_a[k], a);
      read_vector<DT, V>(stage + off_b[k], b);
    }
  }
  // L > 0: to memory.  L = 0: back to the stage, from where `flush` takes it; first, second: whether a vector is to be written.
  __device__ __forceinline__ void write(char* stage, uint64_t out, int k, bool there, const F2 (&a)[kHalf<V>], const F2 (&b)[kHalf<V>], bool first = true,
                                        bool second = true) const {
    if constexpr (L > 0) {
      if (!there) return;
      write_vector<DT, V>((void*)(out + k * L * kBytes), a);
      write_vector<DT, V>((void*)(out + k * L * kBytes + kApart), b);
    } else {
      if (first && off_a[k] < kRowsBytes) write_vector<DT, V>(stage + off_a[k], a);
      if (second && off_b[k] < kRowsBytes) write_vector<DT, V>(stage + off_b[k], b);
    }
  }
  // row: the address of the lane's row, 0 for none
  template <typename S>
  __device__ __forceinline__ void flush(const char* stage, const RopeArgs& a, uint64_t row, const S& to, uint32_t first) const {
    if constexpr (L == 0) {
      using Raw = typename RawOf<kBytes>::T;
      const char* own = stage + (threadIdx.x & 31u) * kBytes;
      __syncwarp();
#pragma unroll
      for (int m = 0; m < kCopies; ++m) {
        const uint64_t at = vector(m, a, row, to, first);
        if (at) *(Raw*)at = *(const Raw*)(own + m * 32 * kBytes);
      }
      __syncwarp();  // before the stage is filled again
    }
  }
};

__device__ __forceinline__ float rsqrt_approx(float x) {  // 2^-22.9 of itself
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Sum over the `lanes` neighbouring lanes of a row, at every one of them.  L = 0: any number of lanes up to 32.
template <int L>
__device__ __forceinline__ float row_sum(F2 two, uint32_t in_row, uint32_t lanes) {
  float v, w;
  f2_unpack(two, v, w);
  v += w;
  if constexpr (L > 0 && (L & (L - 1)) == 0) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  } else if constexpr (L > 0) {
#pragma unroll
    for (uint32_t o = 1; o < L; o <<= 1) {
      w = __shfl_down_sync(0xffffffffu, v, o);
      if (in_row + o < L) v += w;
    }
    return __shfl_sync(0xffffffffu, v, (threadIdx.x & 31u) - in_row);
  } else {
    for (uint32_t o = 1; o < lanes; o <<= 1) {
      w = __shfl_down_sync(0xffffffffu, v, o);
      if (in_row + o < lanes) v += w;
    }
    return __shfl_sync(0xffffffffu, v, (threadIdx.x & 31u) - in_row);
  }
}

// The shared memory of a CTA: the table, the weights in binary32, and for each warp cosines, sines, positions, the addresses that its lanes
// write to, and the ring.
struct Layout {
  uint32_t gamma, warps, warp_bytes, positions, outs, ring;  // byte offsets; the last three within a warp's part
  __host__ __device__ Layout(uint32_t pairs, uint32_t head_dim, int weights, uint32_t group_tokens, uint32_t stages, uint32_t group_bytes) {
    const uint32_t row = (head_dim * 4 + 15) / 16 * 16, half = group_tokens * ((pairs * 4 + 15) / 16 * 16);
    gamma = pairs * 16;
    warps = gamma + weights * row;
    positions = 2 * half;
    outs = positions + (stages + 1) * group_tokens * 16;  // one more: those of the cosines
    ring = outs + stages * 256;
    warp_bytes = ring + stages * group_bytes;
  }
  __host__ __device__ uint32_t bytes() const { return warps + kWarps * warp_bytes; }
};

// The table and the weights into shared memory, by the whole CTA.
__device__ __forceinline__ void stage_table(const RopeArgs& a, char* shared, const Layout& l, const void* g0, const void* g1, int weights) {
#pragma unroll 1
  for (uint32_t i = threadIdx.x; i < a.pairs; i += kThreads) ((ulonglong2*)shared)[i] = ((const ulonglong2*)a.table)[i];
  const uint32_t row = (a.head_dim + 3) / 4 * 4;
  float* gamma = (float*)(shared + l.gamma);
  for (int w = 0; w < weights; ++w) {
    const void* g = w ? g1 : g0;
#pragma unroll 1
    for (uint32_t i = threadIdx.x; i < a.head_dim; i += kThreads) gamma[w * row + i] = g ? load_param(g, i, a.wdt) : 1.0f;
  }
}

// The positions of the group's tokens on the way to a stage, four words for each: its axes', or its place in the sequence.
template <int L, bool MULTI>
__device__ __forceinline__ void copy_positions(const RopeArgs& a, int32_t* to, const Walk<MULTI>& w, const Lane<L, MULTI>& l) {
  if (!l.leads() || !w.there(a)) return;
  to += 4 * l.token;
  if (a.positions) {
    const int32_t* from = a.positions + w.b * a.pos_batch + w.t;
#pragma unroll 1
    for (uint32_t axis = 0; axis < a.axes; ++axis) copy_async<4>(to + axis, from + axis * a.pos_axis);
  } else {
    to[0] = (int32_t)w.t;
  }
}

// The warp's cosines and sines of a group's tokens, from the positions in its stage, unless they are those of the last group, which are kept
// behind the stages'.  True where they are new.
template <int L, bool MULTI>
__device__ __forceinline__ bool warp_phases(const RopeArgs& a, const char* table, const int32_t* at, int32_t* last, const Lane<L, MULTI>& l,
                                            uint32_t group_tokens, bool start, float* cs, float* sn) {
  const uint32_t mine = 4 * (l.on ? l.token : 0);
  const int4 x = *(const int4*)(at + mine), y = *(const int4*)(last + mine);
  if (__all_sync(0xffffffffu, x.x == y.x && x.y == y.y && x.z == y.z && x.w == y.w) && !start) return false;
  if (l.leads()) *(int4*)(last + mine) = x;
  const float sign = a.back ? -1.0f : 1.0f;
  const uint32_t row = (a.pairs + 3) / 4 * 4;
#pragma unroll 1
  for (uint32_t j = threadIdx.x & 31u; j < group_tokens * a.pairs; j += 32) {  // at most 256
    const uint32_t token = (j * a.pairs_inverse) >> 20, i = j - token * a.pairs;
    const ulonglong2 e = ((const ulonglong2*)table)[i];
    const int64_t pos = a.first + at[4 * token + (e.y < a.axes ? (uint32_t)e.y : a.axes - 1)];
    const float2 v = phase(e.x, pos, a.scale, sign);
    cs[token * row + i] = v.x;
    sn[token * row + i] = v.y;
  }
  __syncwarp();
  return true;
}

enum { kPlain = 0, kNorm = 1 };

// A warp's part of the shared memory.
struct Mine {
  float *cs, *sn;
  int32_t* positions;  // of the stages, then those that the cosines are of
  uint64_t* outs;      // the lane's, 32 apart
  char* ring;
  __device__ __forceinline__ Mine(const RopeArgs& a, char* shared, const Layout& lay, uint32_t group_tokens, uint32_t stages) {
    char* mine = shared + lay.warps + (threadIdx.x >> 5) * lay.warp_bytes;
    cs = (float*)mine;
    sn = cs + group_tokens * ((a.pairs + 3) / 4 * 4);
    positions = (int32_t*)(mine + lay.positions);
    outs = (uint64_t*)(mine + lay.outs) + (threadIdx.x & 31u);
    ring = mine + lay.ring;
#pragma unroll 1
    for (uint32_t i = threadIdx.x & 31u; i < (stages + 1) * group_tokens * 4; i += 32) positions[i] = 0;  // those of axes that are not there
    __syncwarp();
  }
};

// Forward of both operators, and the rotation's backward.  The rows of a token are those of its queries' heads, then those of its
// keys'.
template <int DT, int V, int W, bool INTER, int L, bool MULTI, int NORM>
__global__ void __launch_bounds__(kThreads, V == 1 || MULTI ? 2 : 3) rope_kernel(const __grid_constant__ RopeArgs a) {
  constexpr int K = kLaneElems / (2 * V), STAGES = 4;
  using Rows = Group<DT, V, W, K, L, MULTI>;
  extern __shared__ __align__(16) char shared[];
  const uint32_t group_tokens = MULTI ? a.group_tokens[0] : 1;
  const Layout lay(a.pairs, a.head_dim, NORM == kNorm ? 2 : 0, group_tokens, STAGES, Rows::kGroupBytes);
  const uint32_t heads0 = a.heads[0], heads = heads0 + a.heads[1];
  const Lane<L, MULTI> l(a, heads, group_tokens);
  const Places<V, K, INTER, L, MULTI> p(a, l);
  const Rows rows(a, l, p);
  const Mine mine(a, shared, lay, group_tokens, STAGES);
  const uint32_t groups = (heads + l.per - 1) / l.per;
  enter_grid();

  Walk<MULTI> ahead(a, blockIdx.x * kWarps + (threadIdx.x >> 5), 0, groups, l.token);
  Walk<MULTI> now = ahead;  // (several tokens: the addresses to write to come through the ring, and this one only counts)
  bool fresh = true;
  typename Rows::template Source<true> from(a.in[0], a.in[1], heads0, heads), to(a.out[0], a.out[1], heads0, heads);
  const auto fetch = [&](uint32_t stage) {
    if (ahead.left) {
      if (fresh) {
        from.enter(ahead, a.in[0], a.in[1]);
        if (MULTI) to.enter(ahead, a.out[0], a.out[1]);
        copy_positions(a, mine.positions + 4 * stage * group_tokens, ahead, l);
      }
      const uint32_t row = ahead.i * l.per + l.head;
      const bool there = l.on && row < heads && ahead.there(a);
      rows.fetch(mine.ring + stage * Rows::kGroupBytes, a, from, ahead.i * l.per, row, there, l);
      if (MULTI) mine.outs[32 * stage] = there ? to.row(row) : 0;
      fresh = ahead.next(a, 0, groups);
    }
    copy_commit();
  };
#pragma unroll 1
  for (int s = 0; s < STAGES - 1; ++s) fetch(s);
  rows.clear(mine.ring, STAGES);
  stage_table(a, shared, lay, a.gamma[0], a.gamma[1], NORM == kNorm ? 2 : 0);
  __syncthreads();

  Angles<V, K, INTER, L, MULTI> angles;
  bool begins = true, start = true;
  const uint32_t phases = l.token * ((a.pairs + 3) / 4 * 4);
  const float* gamma = (const float*)(shared + lay.gamma);
  const uint32_t gamma_row = (a.head_dim + 3) / 4 * 4;
  for (uint32_t stage = 0; now.left; stage = (stage + 1) % STAGES) {
    copy_wait<STAGES - 2>();
    if (L == 0 || begins) __syncwarp();  // what other lanes copied is here, and the last token's cosines have been read
    if (begins) {
      if (warp_phases(a, shared, mine.positions + 4 * stage * group_tokens, mine.positions + 4 * STAGES * group_tokens, l, group_tokens, start,
                      mine.cs, mine.sn))
        angles.read(p, mine.cs + phases, mine.sn + phases);
      start = false;
      if (!MULTI) to.enter(now, a.out[0], a.out[1]);
    }
    const uint32_t row = now.i * l.per + l.head;
    const uint64_t out = MULTI ? mine.outs[32 * stage] : (L && l.on && row < heads ? to.row(row) : 0);
    char* at = mine.ring + stage * Rows::kGroupBytes;
    F2 fa[K][kHalf<V>], fb[K][kHalf<V>];
#pragma unroll
    for (int k = 0; k < K; ++k) rows.read(at, k, fa[k], fb[k]);
    fetch((stage + STAGES - 1) % STAGES);
    if (NORM == kNorm) {
      F2 sa = f2_both(0.0f), sb = f2_both(0.0f);
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < kHalf<V>; ++j) {
          sa = f2_fma(fa[k][j], fa[k][j], sa);
          sb = f2_fma(fb[k][j], fb[k][j], sb);
        }
      const F2 rstd = f2_both(rsqrt_approx(row_sum<L>(f2_add(sa, sb), l.slot, a.lanes) * a.inv_dim + a.eps));
      const float* weights = gamma + (row >= heads0 ? gamma_row : 0u);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        F2 g[kHalf<V>];
        read_floats<V>(weights + p.at[k], g);
#pragma unroll
        for (int j = 0; j < kHalf<V>; ++j) fa[k][j] = f2_mul(f2_mul(fa[k][j], rstd), g[j]);
        read_floats<V>(weights + p.to[k], g);
#pragma unroll
        for (int j = 0; j < kHalf<V>; ++j) fb[k][j] = f2_mul(f2_mul(fb[k][j], rstd), g[j]);
      }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      angles.turn(p, k, fa[k], fb[k]);
      // without a norm, what does not turn stays in its stage as it came, bit for bit
      rows.write(at, out + l.slot * Rows::kBytes, k, out != 0, fa[k], fb[k], NORM == kNorm || p.turning(k), NORM == kNorm || p.turning2(k));
    }
    rows.flush(at, a, out, to, now.i * l.per);
    begins = MULTI ? now.count(groups) : now.next(a, 0, groups);
  }
}

// The sums of a CTA's rows, `all` (a multiple of eight) of D in shared memory behind which a double a thread has room, by all its threads.  In 64 bits:
// with rows that add up rather than cancel, a chain of some 64 terms in 32 loses several units in the last place.  Narrow rows leave threads for halves or
// quarters of the rows.  Not inlined, as it would change what the kernel holds in registers.
__device__ __noinline__ void add_rows(const float* sums, uint32_t all, uint32_t D, float* out) {
  const uint32_t parts = 4 * D <= kThreads ? 4 : (2 * D <= kThreads ? 2 : 1), of_part = all / parts;
  double* joined = (double*)(sums + all * D);
  for (uint32_t i = threadIdx.x; i < parts * D; i += kThreads) {
    const float* from = sums + i / D * of_part * D + i % D;
    double s = 0.0, t = 0.0;  // an addition waits for the one before it
    for (uint32_t r = 0; r < of_part; r += 2) {
      s += (double)from[r * D];
      t += (double)from[(r + 1) * D];
    }
    if (parts == 1) out[i] = (float)(s + t);
    else joined[i] = s + t;
  }
  if (parts == 1) return;
  __syncthreads();
  if (threadIdx.x < D) {
    double s = 0.0;
    for (uint32_t i = 0; i < parts; ++i) s += joined[i * D + threadIdx.x];
    out[threadIdx.x] = (float)s;
  }
}

// The norm's backward.  A CTA takes rows of queries or of keys only (the first ctas0 CTAs those of queries), so that a lane
// keeps one set of sums for grad_gamma; they are added up over the CTA's rows and left in the scratch, one row of head_dim a CTA.  A lane adds its own rows
// up in 32 bits, which is most of what binary32 weights' gradients are off by: 1.1e-7 for [64, 197, 12 + 12, 64], 3.3e-7 for 2.1 M rows of 128 (with all sums
// in 64 bits 0.7e-7), growing with the root of the rows.
template <int DT, int V, int W, bool INTER, int L, bool MULTI>
__global__ void __launch_bounds__(kThreads, V == 1 ? 1 : 2) qknorm_bwd_kernel(const __grid_constant__ RopeArgs a) {
  constexpr int K = kLaneElems / (2 * V), STAGES = kBwdStages<DT>;
  using Rows = Group<DT, V, W, K, L, MULTI>;
  extern __shared__ __align__(16) char shared[];
  const int which = blockIdx.x >= a.ctas0;
  const uint32_t group_tokens = MULTI ? a.group_tokens[which] : 1;
  const Layout lay(a.pairs, a.head_dim, 1, group_tokens, STAGES, 2 * Rows::kGroupBytes);
  const uint32_t heads = a.heads[which];
  const uint32_t warp = threadIdx.x >> 5;
  const Lane<L, MULTI> l(a, heads, group_tokens);
  const Places<V, K, INTER, L, MULTI> p(a, l);
  const Rows rows(a, l, p);
  const Mine mine(a, shared, lay, group_tokens, STAGES);
  const HeadsArg& x = a.in[which];
  const HeadsArg& g = a.grad[which];
  const HeadsArg& o = a.out[which];
  const uint32_t cta = which ? blockIdx.x - a.ctas0 : blockIdx.x;
  const uint32_t groups = (heads + l.per - 1) / l.per;
  enter_grid();

  Walk<MULTI> ahead(a, cta * kWarps + warp, which, groups, l.token);
  Walk<MULTI> now = ahead;
  bool fresh = true;
  typename Rows::template Source<false> from_x(x, x, heads, heads), from_g(g, g, heads, heads), to(o, o, heads, heads);
  const auto fetch = [&](uint32_t stage) {
    if (ahead.left) {
      if (fresh) {
        from_x.enter(ahead, x, x);
        from_g.enter(ahead, g, g);
        if (MULTI) to.enter(ahead, o, o);
        copy_positions(a, mine.positions + 4 * stage * group_tokens, ahead, l);
      }
      char* at = mine.ring + stage * 2 * Rows::kGroupBytes;
      const uint32_t row = ahead.i * l.per + l.head;
      const bool there = l.on && row < heads && ahead.there(a);
      rows.fetch(at, a, from_x, ahead.i * l.per, row, there, l);
      rows.fetch(at + Rows::kGroupBytes, a, from_g, ahead.i * l.per, row, there, l);
      if (MULTI) mine.outs[32 * stage] = there ? to.row(row) : 0;
      fresh = ahead.next(a, which, groups);
    }
    copy_commit();
  };
#pragma unroll 1
  for (int s = 0; s < STAGES - 1; ++s) fetch(s);
  rows.clear(mine.ring, 2 * STAGES);
  stage_table(a, shared, lay, a.gamma[which], nullptr, 1);
  __syncthreads();

  F2 sa[K][kHalf<V>], sb[K][kHalf<V>];
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int j = 0; j < kHalf<V>; ++j) sa[k][j] = sb[k][j] = f2_both(0.0f);
  bool begins = true, start = true;
  const uint32_t phases = l.token * ((a.pairs + 3) / 4 * 4);
  const float* gamma = (const float*)(shared + lay.gamma);
  for (uint32_t stage = 0; now.left; stage = (stage + 1) % STAGES) {
    copy_wait<STAGES - 2>();
    if (L == 0 || begins) __syncwarp();
    if (begins) {
      warp_phases(a, shared, mine.positions + 4 * stage * group_tokens, mine.positions + 4 * STAGES * group_tokens, l, group_tokens, start, mine.cs,
                  mine.sn);
      start = false;
      if (!MULTI) to.enter(now, o, o);
    }
    Angles<V, K, INTER, L, MULTI> angles;  // read for each group: held over groups they are slower ([4, 4097, 32 + 8, 128] bfloat16 96 us against 93)
    angles.read(p, mine.cs + phases, mine.sn + phases);
    const uint32_t row = now.i * l.per + l.head;
    const uint64_t out = MULTI ? mine.outs[32 * stage] : (L && l.on && row < heads ? to.row(row) : 0);
    const bool there = MULTI ? out != 0 : l.on && row < heads;
    F2 xa[K][kHalf<V>], xb[K][kHalf<V>], ua[K][kHalf<V>], ub[K][kHalf<V>];
    char* at = mine.ring + stage * 2 * Rows::kGroupBytes;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      rows.read(at, k, xa[k], xb[k]);
      rows.read(at + Rows::kGroupBytes, k, ua[k], ub[k]);
    }
    fetch((stage + STAGES - 1) % STAGES);
    F2 sum = f2_both(0.0f), other = f2_both(0.0f);
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int j = 0; j < kHalf<V>; ++j) {
        sum = f2_fma(xa[k][j], xa[k][j], sum);
        other = f2_fma(xb[k][j], xb[k][j], other);
      }
    // a row that does not exist is zeros in x and in the gradient: with this rstd it adds nothing to any sum
    float root = rsqrt_approx(row_sum<L>(f2_add(sum, other), l.slot, a.lanes) * a.inv_dim + a.eps);
    if (!there) root = 0.0f;
    const F2 rstd = f2_both(root);
    sum = other = f2_both(0.0f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      angles.turn(p, k, ua[k], ub[k]);
      F2 w[kHalf<V>];
      read_floats<V>(gamma + p.at[k], w);
#pragma unroll
      for (int j = 0; j < kHalf<V>; ++j) {
        xa[k][j] = f2_mul(xa[k][j], rstd);  // xhat
        sa[k][j] = f2_fma(ua[k][j], xa[k][j], sa[k][j]);
        ua[k][j] = f2_mul(ua[k][j], w[j]);
        sum = f2_fma(ua[k][j], xa[k][j], sum);
      }
      read_floats<V>(gamma + p.to[k], w);
#pragma unroll
      for (int j = 0; j < kHalf<V>; ++j) {
        xb[k][j] = f2_mul(xb[k][j], rstd);
        sb[k][j] = f2_fma(ub[k][j], xb[k][j], sb[k][j]);
        ub[k][j] = f2_mul(ub[k][j], w[j]);
        other = f2_fma(ub[k][j], xb[k][j], other);
      }
    }
    const F2 mean = f2_both(-row_sum<L>(f2_add(sum, other), l.slot, a.lanes) * a.inv_dim);
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int j = 0; j < kHalf<V>; ++j) {
        ua[k][j] = f2_mul(f2_fma(mean, xa[k][j], ua[k][j]), rstd);
        ub[k][j] = f2_mul(f2_fma(mean, xb[k][j], ub[k][j]), rstd);
      }
      rows.write(at, out + l.slot * Rows::kBytes, k, out != 0, ua[k], ub[k]);
    }
    rows.flush(at, a, out, to, now.i * l.per);
    begins = MULTI ? now.count(groups) : now.next(a, which, groups);
  }
  if (!a.partials) return;
  copy_wait<0>();
  __syncthreads();  // the rings' place becomes the sums'
  const uint32_t D = a.head_dim, held = l.per * group_tokens, all = kWarps * held;  // rows with sums
  float* sums = (float*)(shared + lay.warps);
  if (l.on) {
    float* own = sums + (warp * held + l.row) * D;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int j = 0; j < kHalf<V>; ++j) {
        float u, v;
        f2_unpack(sa[k][j], u, v);
        if (p.has_first(k)) {
          own[p.at[k] + 2 * j] = u;
          if (V > 1) own[p.at[k] + 2 * j + 1] = v;
        }
        f2_unpack(sb[k][j], u, v);
        if (p.has_second(k)) {
          own[p.to[k] + 2 * j] = u;
          if (V > 1) own[p.to[k] + 2 * j + 1] = v;
        }
      }
  }
  __syncthreads();
  add_rows(sums, all, D, a.partials + (uint64_t)blockIdx.x * D);
}

template <int DT, int V, int W, bool INTER, int L, bool MULTI>
cudaError_t launch_one(int mode, const RopeArgs& a, unsigned grid, cudaStream_t st) {
  static std::atomic<uint64_t> ready[3] = {};
  const bool bwd = mode == kRopeBwdNorm;
  constexpr uint32_t group = Group<DT, V, W, kLaneElems / (2 * V), L, MULTI>::kGroupBytes;
  // the sums of the backward pass take the rings' place: 16 floats a lane, and one double a thread
  static_assert(kBwdStages<DT> * 2 * group >= 32 * (kLaneElems * sizeof(float) + sizeof(double)), "the sums fit in the rings");
  const int weights = mode == kRopeFwdNorm ? 2 : (bwd ? 1 : 0);
  const uint32_t stages = bwd ? kBwdStages<DT> : 4, bytes = bwd ? 2 * group : group;
  const size_t smem = std::max(Layout(a.pairs, a.head_dim, weights, a.group_tokens[0], stages, bytes).bytes(),
                               bwd ? Layout(a.pairs, a.head_dim, weights, a.group_tokens[1], stages, bytes).bytes() : 0u);
  // the leave is asked for once, for any shape: at most 256 pairs, 32 tokens and 512 elements
  const size_t most = Layout(kMaxHeadDim / 2, kMaxHeadDim, weights, 1, stages, bytes).bytes() + kWarps * 32 * 16 * (stages + 1);
  const auto go = [&](void (*kernel)(const RopeArgs)) {
    const cudaError_t e = allow_shared(kernel, most, ready[mode]);
    return e != cudaSuccess ? e : launch_overlapped(kernel, dim3(grid), kThreads, smem, st, a);
  };
  if (bwd) return go(qknorm_bwd_kernel<DT, V, W, INTER, L, MULTI>);
  return mode == kRopeFwdNorm ? go(rope_kernel<DT, V, W, INTER, L, MULTI, kNorm>) : go(rope_kernel<DT, V, W, INTER, L, MULTI, kPlain>);
}

template <int DT, int V, int W, int L, bool MULTI>
cudaError_t launch_layout(int mode, const RopeArgs& a, unsigned grid, cudaStream_t st) {
  if constexpr (V > 1)
    if (a.interleaved) return launch_one<DT, V, W, true, L, MULTI>(mode, a, grid, st);
  return launch_one<DT, V, W, false, L, MULTI>(mode, a, grid, st);
}

}  // namespace

#if defined(S2A_ROPE_WHOLE_ROWS)
template <int DT>
cudaError_t launch_rope_whole(int mode, const RopeArgs& a, unsigned grid, cudaStream_t st) {
  constexpr int W = 16 / Io<DT>::kBytes;  // the widest vector
  switch (a.head_dim) {
    case 32: return launch_layout<DT, W, W, 2, false>(mode, a, grid, st);
    case 64: return launch_layout<DT, W, W, 4, false>(mode, a, grid, st);
    case 96: return launch_layout<DT, W, W, 6, false>(mode, a, grid, st);
    case 128: return launch_layout<DT, W, W, 8, false>(mode, a, grid, st);
    case 160: return launch_layout<DT, W, W, 10, false>(mode, a, grid, st);
    case 192: return launch_layout<DT, W, W, 12, false>(mode, a, grid, st);
    default: return launch_layout<DT, W, W, 16, false>(mode, a, grid, st);
  }
}
#else
// (V, W) is one of these: W the widest vector, or both 2 or 1.
template <int DT, bool MULTI>
cudaError_t launch_rope_any(int mode, uint32_t V, uint32_t W, const RopeArgs& a, unsigned grid, cudaStream_t st) {
  constexpr int M = 16 / Io<DT>::kBytes;
  if (W == 1) return launch_layout<DT, 1, 1, 0, MULTI>(mode, a, grid, st);
  if (W == 2) return launch_layout<DT, 2, 2, 0, MULTI>(mode, a, grid, st);
  if (V == 1) return launch_layout<DT, 1, M, 0, MULTI>(mode, a, grid, st);
  if (V == 2) return launch_layout<DT, 2, M, 0, MULTI>(mode, a, grid, st);
  if constexpr (M == 8)
    if (V == 4) return launch_layout<DT, 4, M, 0, MULTI>(mode, a, grid, st);
  return launch_layout<DT, M, M, 0, MULTI>(mode, a, grid, st);
}
#endif

}  // namespace s2a
