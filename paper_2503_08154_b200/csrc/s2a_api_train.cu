// extern "C" entry points around the scores and after the backward pass: argument checks and launches of rotary positions,
// the norms of queries and keys, the AdamW step and the gradients' norm.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>

#include "../../include/s2a.h"
#include "s2a_common.cuh"
#include "s2a_launch.h"

namespace {

using namespace s2a;

bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }
bool bad_dtype(int dt) { return dt != S2A_F32 && dt != S2A_BF16; }
size_t elem_bytes(int dt) { return dt == S2A_F32 ? 4 : 2; }

// ---- tensors of heads: rows of `row` bytes over up to three dimensions, the widest stride first
struct Rows {
  int dims;
  size_t n[3], s[3];  // extents above 1, strides in bytes
  size_t row;
  size_t extent(int from) const {  // bytes from the first row's start to the last row's end
    size_t e = row;
    for (int i = from; i < dims; ++i) e += (n[i] - 1) * s[i];
    return e;
  }
};

constexpr size_t kMaxExtent = (size_t)1 << 60;

// false where the rows cannot be addressed
bool make_rows(const size_t* strides, size_t batch, size_t tokens, size_t heads, size_t head_dim, size_t es, Rows& r) {
  const size_t n[3] = {batch, tokens, heads};
  r.dims = 0;
  r.row = head_dim * es;
  size_t extent = r.row;
  for (int i = 0; i < 3; ++i) {
    if (n[i] <= 1) continue;
    if (i == 2 && strides[i] >> 32) return false;  // the kernels hold a head's stride in 32 bits
    if (strides[i] != 0 && n[i] - 1 > (kMaxExtent - extent) / es / strides[i]) return false;
    extent += (n[i] - 1) * strides[i] * es;
    int at = r.dims++;
    for (; at > 0 && r.s[at - 1] < strides[i] * es; --at) {
      r.n[at] = r.n[at - 1];
      r.s[at] = r.s[at - 1];
    }
    r.n[at] = n[i];
    r.s[at] = strides[i] * es;
  }
  return true;
}

// Whether rows of one tensor lie on one another: each stride must step over all that it holds.
bool folds(const Rows& r) {
  for (int i = 0; i < r.dims; ++i)
    if (r.s[i] < r.extent(i + 1)) return true;
  return false;
}

// Whether rows of a and b, whose first row starts `delta` bytes after a's, can meet.  Where both step by one widest stride that
// holds all the rest, only the offsets of one step matter; otherwise the whole extents are compared.
bool rows_meet(const Rows& a, int ia, const Rows& b, int ib, long long delta) {
  const long long ea = (long long)a.extent(ia), eb = (long long)b.extent(ib);
  if (delta >= ea || -delta >= eb) return false;
  if (ia < a.dims && ib < b.dims && a.s[ia] == b.s[ib]) {
    const long long s = (long long)a.s[ia];
    if (s >= (long long)a.extent(ia + 1) && s >= (long long)b.extent(ib + 1)) {
      long long d = delta % s;
      if (d < 0) d += s;
      for (int i = 0; i < 2; ++i, d -= s) {
        const long long steps = (d - delta) / s;  // of b forward, or of a
        if (steps < -(long long)(a.n[ia] - 1) || steps > (long long)(b.n[ib] - 1)) continue;
        if (rows_meet(a, ia + 1, b, ib + 1, d)) return true;
      }
      return false;
    }
  }
  return true;
}

// Whether each row of the one is that of the other.
bool same_place(const HeadsArg& a, const HeadsArg& b) {
  return a.data == b.data && a.batch == b.batch && a.token == b.token && a.head == b.head;
}

bool tensors_meet(const void* pa, const Rows& a, const void* pb, const Rows& b) {
  return rows_meet(a, 0, b, 0, (long long)((uintptr_t)pb - (uintptr_t)pa));
}

int run_rope(const s2a_rope_args* args, int mode, int back, void* stream) {
  if (!args) return S2A_ERR_NULL;
  const s2a_rope_args& c = *args;
  const bool norm = mode != kRopePlain, bwd = mode == kRopeBwdNorm;
  const size_t heads[2] = {c.heads_q, c.heads_k};
  if (bad_dtype(c.dt) || (norm && bad_dtype(c.wdt))) return S2A_ERR_DTYPE;
  if (c.head_dim == 0 || c.head_dim > kMaxHeadDim || c.rot_dim % 2 != 0 || c.rot_dim > c.head_dim || (!norm && c.rot_dim == 0) ||
      heads[0] > 65535u || heads[1] > 65535u || c.batch > 0x7fffffffull || c.tokens > 0x7fffffffull ||
      c.batch * c.tokens > 0x7fffffffull || (c.rot_dim && (c.axes == 0 || c.axes > kMaxAxes)))
    return S2A_ERR_SHAPE;
  if (!(fabsf(c.scale) <= 3.4028234e38f) || (norm && !(c.eps >= 0.0f && c.eps <= 3.4028234e38f))) return S2A_ERR_VALUE;
  const void* const in[2] = {c.q, c.k};
  const void* const grad[2] = {c.grad_q, c.grad_k};
  void* const out[2] = {c.out_q, c.out_k};
  // weights of heads that are not there are not looked at, and not read by the kernels
  const void* const gamma[2] = {norm && c.heads_q ? c.gamma_q : nullptr, norm && c.heads_k ? c.gamma_k : nullptr};
  void* const sums[2] = {bwd ? c.grad_gamma_q : nullptr, bwd ? c.grad_gamma_k : nullptr};
  const size_t* const in_stride[2] = {c.q_stride, c.k_stride};
  const size_t* const grad_stride[2] = {c.grad_q_stride, c.grad_k_stride};
  const size_t* const out_stride[2] = {c.out_q_stride, c.out_k_stride};
  const size_t es = elem_bytes(c.dt), ws = norm ? elem_bytes(c.wdt) : 1;
  const bool empty = c.batch * c.tokens == 0 || heads[0] + heads[1] == 0;
  for (int i = 0; i < 2; ++i)
    if (misaligned(gamma[i], ws) || misaligned(sums[i], ws)) return S2A_ERR_ALIGN;
  if (!empty) {
    if ((c.rot_dim && (!c.table || (!c.positions && c.axes > 1))) || ((sums[0] || sums[1]) && !c.scratch)) return S2A_ERR_NULL;
    if ((c.rot_dim && (misaligned(c.table, 16) || misaligned(c.positions, 4))) || (bwd && misaligned(c.scratch, 16))) return S2A_ERR_ALIGN;
    if (c.rot_dim && c.positions && (c.pos_batch_stride > kMaxExtent / 0x7fffffffull || c.pos_axis_stride > kMaxExtent / kMaxAxes))
      return S2A_ERR_SHAPE;
  }
  RopeArgs a = {};
  Rows wrote[2], had[4];
  const HeadsArg* had_by[4];
  int had_side[4], n = 0;  // queries' or keys'
  for (int i = 0; i < 2 && !empty; ++i) {
    if (heads[i] == 0) continue;
    if (!in[i] || !out[i] || (bwd && !grad[i])) return S2A_ERR_NULL;
    if (misaligned(in[i], es) || misaligned(out[i], es) || (bwd && misaligned(grad[i], es))) return S2A_ERR_ALIGN;
    const auto take = [&](const void* p, const size_t* s, HeadsArg& h, Rows& r) {
      // a dimension of one has no stride
      h = HeadsArg{p, c.batch > 1 ? s[0] : 0, c.tokens > 1 ? s[1] : 0, heads[i] > 1 ? s[2] : 0};
      return make_rows(s, c.batch, c.tokens, heads[i], c.head_dim, es, r);
    };
    had_by[n] = &a.in[i];
    had_side[n] = i;
    if (!take(in[i], in_stride[i], a.in[i], had[n++])) return S2A_ERR_SHAPE;
    if (bwd) {
      had_by[n] = &a.grad[i];
      had_side[n] = i;
      if (!take(grad[i], grad_stride[i], a.grad[i], had[n++])) return S2A_ERR_SHAPE;
    }
    if (!take(out[i], out_stride[i], a.out[i], wrote[i]) || folds(wrote[i])) return S2A_ERR_SHAPE;
    a.heads[i] = (uint32_t)heads[i];
  }
  for (int i = 0; i < 2 && !empty; ++i) {
    if (heads[i] == 0) continue;
    for (int j = 0; j < n; ++j) {
      // in place: a warp has read a row of the output's own input before it writes there; the other side's it reads at any time
      if (had_side[j] == i && same_place(*had_by[j], a.out[i])) continue;
      if (tensors_meet(had_by[j]->data, had[j], out[i], wrote[i])) return S2A_ERR_OVERLAP;
    }
    if (i == 1 && heads[0] && tensors_meet(out[0], wrote[0], out[1], wrote[1])) return S2A_ERR_OVERLAP;
  }
  a.gamma[0] = gamma[0];
  a.gamma[1] = gamma[1];
  a.positions = c.rot_dim ? c.positions : nullptr;
  a.table = c.table;
  a.first = a.positions ? 0 : c.first;
  a.pos_axis = c.pos_axis_stride;
  a.pos_batch = c.pos_batch_stride;
  a.batch = (uint32_t)c.batch;
  a.tokens = (uint32_t)c.tokens;
  a.head_dim = (uint32_t)c.head_dim;
  a.pairs = (uint32_t)(c.rot_dim / 2);
  a.axes = c.rot_dim ? (uint32_t)c.axes : 1u;
  a.interleaved = c.interleaved != 0;
  a.back = back;
  a.wdt = c.wdt;
  a.scale = c.scale;
  a.eps = c.eps;
  return launch_rope(mode, c.dt, a, sums[0], sums[1], (float*)c.scratch, (cudaStream_t)stream) == cudaSuccess ? S2A_OK : S2A_ERR_CUDA;
}

// ---- the plan of a step
struct Span {
  uintptr_t from, to;
  bool written;
};

size_t blocks_of(size_t n) { return (n + kStepBlock - 1) / kStepBlock; }

// Blocks of a chunk: one where the plan is small, so that every warp gets one; four where every warp gets a chunk all the same, and sixteen where it
// gets sixteen, as each chunk costs a look at the plan and a wait for its first block (302 M weights with 8-bit states, before each operation was rounded: 608 us with
// 16 blocks, 698 with 4; their gradients' norm 90 and 105).
size_t chunk_blocks_of(size_t blocks) {
  const size_t warps = 148 * 20;
  return blocks >= 256 * warps ? 16 : (blocks >= 4 * warps ? 4 : 1);
}

// The plan's chunks, and blocks of a chunk; 0 where there are too many.
size_t count_chunks(const s2a_step_tensor* tensors, size_t n_tensors, size_t& chunk_blocks) {
  size_t blocks = 0, chunks = 0;
  for (size_t i = 0; i < n_tensors; ++i) {
    if (tensors[i].n > kMaxExtent) return 0;
    blocks += blocks_of(tensors[i].n);
    if (blocks > ((size_t)1 << 40)) return 0;
  }
  chunk_blocks = chunk_blocks_of(blocks);
  for (size_t i = 0; i < n_tensors; ++i) chunks += (blocks_of(tensors[i].n) + chunk_blocks - 1) / chunk_blocks;
  return chunks > 0x7fffffffull ? 0 : chunks;
}

// Elements before the first that lies on the 16-byte grid in all of a tensor's parts, or kStepScalar.  Eight elements are whole
// vectors in every type.
uint32_t common_head(const void* const* p, const size_t* bytes, int parts) {
  for (uint32_t h = 0; h < 8; ++h) {
    bool ok = true;
    for (int i = 0; i < parts && ok; ++i) ok = ((uintptr_t)p[i] + h * bytes[i]) % std::min<size_t>(16, 8 * bytes[i]) == 0;
    if (ok) return h;
  }
  return kStepScalar;
}

bool bad_rate(float v) { return !(v >= 0.0f && v <= 3.4028234e38f); }

int bad_plan(const s2a_step_plan* plan, const void* image) {
  if (!plan) return S2A_ERR_NULL;
  if (plan->n_chunks && !image) return S2A_ERR_NULL;
  if (misaligned(image, 16)) return S2A_ERR_ALIGN;
  if (plan->n_chunks > 0x7fffffffull || plan->n_tensors > 0x7fffffffull || plan->chunk_blocks > 16) return S2A_ERR_SHAPE;
  return S2A_OK;
}

StepArgs step_args(const s2a_step_plan* plan, const void* image, const float* control) {
  StepArgs a = {};
  a.tensors = (const StepTensor*)image;
  a.owner = (const uint32_t*)((const char*)image + plan->n_tensors * sizeof(StepTensor));
  a.n_chunks = (uint32_t)plan->n_chunks;
  a.chunk_blocks = (uint32_t)plan->chunk_blocks;
  a.control = control;
  return a;
}

}  // namespace

extern "C" {

int s2a_rope_fwd(const s2a_rope_args* args, void* cuda_stream) { return run_rope(args, kRopePlain, 0, cuda_stream); }
int s2a_rope_bwd(const s2a_rope_args* args, void* cuda_stream) { return run_rope(args, kRopePlain, 1, cuda_stream); }
int s2a_qknorm_rope_fwd(const s2a_rope_args* args, void* cuda_stream) { return run_rope(args, kRopeFwdNorm, 0, cuda_stream); }
int s2a_qknorm_rope_bwd(const s2a_rope_args* args, void* cuda_stream) { return run_rope(args, kRopeBwdNorm, 1, cuda_stream); }

size_t s2a_qknorm_rope_scratch_bytes(size_t, size_t, size_t, size_t, size_t head_dim) {
  return head_dim == 0 || head_dim > kMaxHeadDim ? 0 : (size_t)qknorm_scratch_bytes((uint32_t)head_dim);
}

int s2a_rope_table(uint64_t* table, size_t rot_dim, double base, int scaling, double factor, double original_length, double slow,
                   double fast, size_t axes) {
  const size_t pairs = rot_dim / 2;
  if (rot_dim % 2 != 0 || rot_dim > kMaxHeadDim || axes == 0 || axes > kMaxAxes || pairs % axes != 0) return S2A_ERR_SHAPE;
  if (!(base >= 1.0) || isinf(base) || scaling < kRopeScaleNone || scaling > kRopeScaleParts) return S2A_ERR_VALUE;
  if (scaling != kRopeScaleNone && (!(factor > 0.0) || isinf(factor))) return S2A_ERR_VALUE;
  if (scaling == kRopeScaleParts &&
      (!(original_length > 0.0) || isinf(original_length) || !(slow >= 0.0) || !(fast > slow) || isinf(fast)))
    return S2A_ERR_VALUE;
  if (pairs == 0) return S2A_OK;
  if (!table) return S2A_ERR_NULL;
  if (misaligned(table, 8)) return S2A_ERR_ALIGN;
  rope_table(table, (uint32_t)pairs, base, scaling, factor, original_length, slow, fast, (uint32_t)axes);
  return S2A_OK;
}

size_t s2a_step_plan_bytes(const s2a_step_tensor* tensors, size_t n_tensors) {
  if (!tensors || n_tensors > 0x7fffffffull) return 0;
  size_t chunk_blocks;
  return n_tensors * sizeof(StepTensor) + count_chunks(tensors, n_tensors, chunk_blocks) * sizeof(uint32_t);
}

int s2a_step_plan_fill(const s2a_step_tensor* tensors, size_t n_tensors, int pdt, int gdt, int state_bits, void* image,
                       s2a_step_plan* plan) {
  if (!plan || (n_tensors && (!tensors || !image))) return S2A_ERR_NULL;
  if (n_tensors > 0x7fffffffull) return S2A_ERR_SHAPE;
  bool grads_only = n_tensors > 0;
  for (size_t i = 0; i < n_tensors; ++i) grads_only = grads_only && !tensors[i].param;
  if (bad_dtype(gdt) || (!grads_only && bad_dtype(pdt))) return S2A_ERR_DTYPE;
  if (!grads_only && state_bits != 8 && state_bits != 32) return S2A_ERR_VALUE;
  size_t chunk_blocks = 1, elems = 0;
  for (size_t i = 0; i < n_tensors; ++i) elems |= tensors[i].n;
  if (count_chunks(tensors, n_tensors, chunk_blocks) == 0 && elems) return S2A_ERR_SHAPE;
  if (misaligned(image, 16)) return S2A_ERR_ALIGN;
  const size_t ps = elem_bytes(pdt), gs = elem_bytes(gdt), ss = state_bits == 8 ? 1 : 4;
  for (size_t i = 0; i < n_tensors; ++i) {
    const s2a_step_tensor& t = tensors[i];
    if (t.n == 0) continue;
    if (!t.grad) return S2A_ERR_NULL;
    if (misaligned(t.grad, gs)) return S2A_ERR_ALIGN;
    if (grads_only) continue;
    if (!t.param || !t.exp_avg || !t.exp_avg_sq || (state_bits == 8 && (!t.exp_avg_scale || !t.exp_avg_sq_scale))) return S2A_ERR_NULL;
    if (t.copy && pdt != S2A_F32) return S2A_ERR_DTYPE;
    if (misaligned(t.param, ps) || misaligned(t.exp_avg, ss) || misaligned(t.exp_avg_sq, ss) || misaligned(t.copy, 2) ||
        (state_bits == 8 && (misaligned(t.exp_avg_scale, 4) || misaligned(t.exp_avg_sq_scale, 4))))
      return S2A_ERR_ALIGN;
    if (bad_rate(t.weight_decay) || bad_rate(t.lr_scale)) return S2A_ERR_VALUE;
  }
  if (!grads_only && n_tensors) {  // what is written lies on nothing else
    Span* spans = (Span*)malloc(n_tensors * 7 * sizeof(Span));
    if (!spans) return S2A_ERR_MEMORY;
    size_t count = 0;
    const auto add = [&](const void* p, size_t bytes, bool written) {
      if (p && bytes) spans[count++] = Span{(uintptr_t)p, (uintptr_t)p + bytes, written};
    };
    for (size_t i = 0; i < n_tensors; ++i) {
      const s2a_step_tensor& t = tensors[i];
      const size_t blocks = blocks_of(t.n);
      add(t.param, t.n * ps, true);
      add(t.grad, t.n * gs, false);
      add(t.exp_avg, t.n * ss, true);
      add(t.exp_avg_sq, t.n * ss, true);
      add(t.copy, t.n * 2, true);
      if (state_bits == 8) {
        add(t.exp_avg_scale, blocks * 4, true);
        add(t.exp_avg_sq_scale, blocks * 4, true);
      }
    }
    std::sort(spans, spans + count, [](const Span& x, const Span& y) { return x.from < y.from; });
    uintptr_t written = 0, any = 0;  // the furthest ends so far
    bool meet = false;
    for (size_t i = 0; i < count && !meet; ++i) {
      meet = spans[i].from < (spans[i].written ? any : written);
      any = std::max(any, spans[i].to);
      if (spans[i].written) written = std::max(written, spans[i].to);
    }
    free(spans);
    if (meet) return S2A_ERR_OVERLAP;
  }
  StepTensor* out = (StepTensor*)image;
  uint32_t* owner = (uint32_t*)((char*)image + n_tensors * sizeof(StepTensor));
  uint32_t chunk = 0;
  uint64_t block = 0;
  for (size_t i = 0; i < n_tensors; ++i) {
    const s2a_step_tensor& t = tensors[i];
    StepTensor& o = out[i];
    memset(&o, 0, sizeof o);
    o.g = t.grad;
    o.n = t.n;
    o.chunk0 = chunk;
    o.block0 = block;
    const void* parts[5] = {t.grad, t.param, t.exp_avg, t.exp_avg_sq, t.copy};
    const size_t bytes[5] = {gs, ps, ss, ss, 2};
    o.head = t.n == 0 ? 0 : common_head(parts, bytes, grads_only ? 1 : (t.copy ? 5 : 4));
    if (!grads_only) {
      o.p = t.param;
      o.m = t.exp_avg;
      o.v = t.exp_avg_sq;
      o.copy = t.copy;
      o.decay = t.weight_decay;
      o.lr = t.lr_scale;
      if (state_bits == 8) {
        o.m_scale = t.exp_avg_scale;
        o.v_scale = t.exp_avg_sq_scale;
      }
    }
    block += blocks_of(t.n);
    for (size_t c = (blocks_of(t.n) + chunk_blocks - 1) / chunk_blocks; c > 0; --c) owner[chunk++] = (uint32_t)i;
  }
  plan->bytes = n_tensors * sizeof(StepTensor) + (size_t)chunk * sizeof(uint32_t);
  plan->n_tensors = n_tensors;
  plan->n_chunks = chunk;
  plan->chunk_blocks = chunk_blocks;
  plan->pdt = pdt;
  plan->gdt = gdt;
  plan->state_bits = state_bits;
  plan->grads_only = grads_only;
  return S2A_OK;
}

int s2a_adamw_step(const s2a_step_plan* plan, const void* image, const float* control, const float* clip, const uint64_t* rng,
                   uint64_t site, double beta1, double beta2, double eps, void* cuda_stream) {
  const int bad = bad_plan(plan, image);
  if (bad) return bad;
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0 && eps <= 3.4028234e38)) return S2A_ERR_VALUE;
  if (plan->n_chunks == 0) return S2A_OK;
  if (plan->grads_only || !control) return S2A_ERR_NULL;
  if (misaligned(control, 4) || misaligned(clip, 4) || misaligned(rng, 8)) return S2A_ERR_ALIGN;
  StepArgs a = step_args(plan, image, control);
  a.clip = clip;
  a.rng = rng;
  a.site = site;
  a.beta1 = (float)beta1;
  a.beta2 = (float)beta2;
  a.one_beta1 = (float)(1.0 - beta1);
  a.one_beta2 = (float)(1.0 - beta2);
  a.root_one_beta2 = (float)sqrt(1.0 - beta2);
  a.log_beta1 = (float)log(beta1);
  a.log_beta2 = (float)log(beta2);
  a.eps = (float)eps;
  return launch_adamw(plan->pdt, plan->gdt, plan->state_bits, a, (cudaStream_t)cuda_stream) == cudaSuccess ? S2A_OK : S2A_ERR_CUDA;
}

size_t s2a_grad_norm_scratch_bytes(const s2a_step_plan* plan) {
  return !plan || plan->n_chunks > 0x7fffffffull ? 0 : (size_t)grad_norm_scratch_bytes((uint32_t)plan->n_chunks);
}

int s2a_grad_norm(const s2a_step_plan* plan, const void* image, const float* control, double max_norm, float* clip, void* scratch,
                  void* cuda_stream) {
  const int bad = bad_plan(plan, image);
  if (bad) return bad;
  if (!(max_norm >= 0.0)) return S2A_ERR_VALUE;
  if (!control || !clip || !scratch) return S2A_ERR_NULL;
  if (misaligned(control, 4) || misaligned(clip, 4) || misaligned(scratch, 16)) return S2A_ERR_ALIGN;
  return launch_grad_norm(plan->gdt, step_args(plan, image, control), (float)max_norm, clip, (double*)scratch,
                          (cudaStream_t)cuda_stream) == cudaSuccess ? S2A_OK : S2A_ERR_CUDA;
}

}  // extern "C"
