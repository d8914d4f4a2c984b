// extern "C" entry points of libs2a.so: argument checks, choice of kernel path, launch.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include "../../include/s2a.h"
#include "s2a_common.cuh"
#include "s2a_launch.h"

namespace {

using namespace s2a;

bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

int check_args(const void* a, const void* b, const void* codes, const void* meta, size_t n,
               size_t row_len, int dt) {
  if (dt != S2A_F32 && dt != S2A_BF16) return S2A_ERR_DTYPE;
  if (row_len == 0 || row_len > 0x7fffffffull || n % row_len != 0) return S2A_ERR_SHAPE;
  if (n == 0) return S2A_OK;
  if (!a || !b || !codes || !meta) return S2A_ERR_NULL;
  if (misaligned(a, 16) || misaligned(b, 16) || misaligned(codes, 16) || misaligned(meta, 8))
    return S2A_ERR_ALIGN;
  // in-place (a == b) is fine: every element, and every row, is read before it is written;
  // an output that merely overlaps its input would be overwritten while still unread
  if (a != b) {
    const uintptr_t bytes = (uintptr_t)n * (dt == S2A_F32 ? 4u : 2u);
    const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
    if (pa < pb + bytes && pb < pa + bytes) return S2A_ERR_OVERLAP;
  }
  return S2A_OK;
}

// Full tiles go to the pipelined kernel, whatever rows remain to the row-at-a-time one.
int run(int kernel, const void* in, void* out, uint8_t* codes, float* meta, size_t n,
        size_t row_len, int dt, void* stream) {
  int rc = check_args(in, out, codes, meta, n, row_len, dt);
  if (rc != S2A_OK || n == 0) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  const uint64_t n_rows = n / row_len;
  TilePlan p = plan_tile(kernel, dt, n_rows, (uint32_t)row_len);
  uint64_t done_rows = 0;
  // the pipelined path moves metadata with 16-byte bulk copies
  if (p.tile_rows != 0 && p.n_tiles != 0 && !misaligned(meta, 16)) {
    TileArgs ta{in, out, codes, meta, (uint32_t)row_len, p.n_tiles};
    if (launch_tile(kernel, dt, p, ta, st) != cudaSuccess) return S2A_ERR_CUDA;
    done_rows = p.n_tiles * p.tile_rows;
  }
  if (done_rows < n_rows) {
    RowwiseArgs ra{in, out, codes, meta, done_rows, n_rows - done_rows, (uint32_t)row_len};
    if (launch_rowwise(kernel, dt, ra, st) != cudaSuccess) return S2A_ERR_CUDA;
  }
  return S2A_OK;
}

}  // namespace

extern "C" {

size_t s2a_codes_bytes(size_t n_elems) { return (n_elems + 1) / 2; }

size_t s2a_meta_bytes(size_t n_elems, size_t row_len) {
  return row_len == 0 ? 0 : (n_elems / row_len) * 2 * sizeof(float);
}

const char* s2a_status_string(int status) {
  switch (status) {
    case S2A_OK: return "S2A_OK";
    case S2A_ERR_NULL: return "S2A_ERR_NULL: a required pointer is NULL";
    case S2A_ERR_SHAPE: return "S2A_ERR_SHAPE: row_len is 0 or does not divide n_elems";
    case S2A_ERR_ALIGN: return "S2A_ERR_ALIGN: data/codes need 16-byte, meta 8-byte alignment";
    case S2A_ERR_DTYPE: return "S2A_ERR_DTYPE: dt must be S2A_F32 or S2A_BF16";
    case S2A_ERR_CUDA: return "S2A_ERR_CUDA: the CUDA runtime refused the launch";
    case S2A_ERR_DEVICE: return "S2A_ERR_DEVICE: a kernel gave up on a bounded wait";
    case S2A_ERR_TOO_LARGE:
      return "S2A_ERR_TOO_LARGE: n_elems exceeds the built-in scratch of the allocation-free entry point "
             "(536,870,912 elements); use s2a_gelu_fwd_tensor_range with your own scratch";
    case S2A_ERR_OVERLAP: return "S2A_ERR_OVERLAP: the output overlaps the input without being the same tensor";
    case S2A_ERR_VALUE: return "S2A_ERR_VALUE: a scalar argument is outside its range";
    case S2A_ERR_MEMORY: return "S2A_ERR_MEMORY: the host has no memory for a plan's checks";
    default: return "unknown s2a status";
  }
}

int s2a_gelu_fwd(const void* x, void* y, uint8_t* codes, float* meta, size_t n_elems,
                 size_t row_len, int dt, void* cuda_stream) {
  return run(kGeluFwd, x, y, codes, meta, n_elems, row_len, dt, cuda_stream);
}

int s2a_gelu_bwd(const void* grad_out, const uint8_t* codes, const float* meta, void* grad_in,
                 size_t n_elems, size_t row_len, int dt, void* cuda_stream) {
  return run(kGeluBwd, grad_out, grad_in, const_cast<uint8_t*>(codes), const_cast<float*>(meta),
             n_elems, row_len, dt, cuda_stream);
}

int s2a_softmax_fwd(const void* x, void* y, uint8_t* codes, float* meta, size_t n_elems,
                    size_t row_len, int dt, void* cuda_stream) {
  return run(kSoftmaxFwd, x, y, codes, meta, n_elems, row_len, dt, cuda_stream);
}

int s2a_softmax_bwd(const void* grad_out, const uint8_t* codes, const float* meta, void* grad_in,
                    size_t n_elems, size_t row_len, int dt, void* cuda_stream) {
  return run(kSoftmaxBwd, grad_out, grad_in, const_cast<uint8_t*>(codes),
             const_cast<float*>(meta), n_elems, row_len, dt, cuda_stream);
}

static int run_cap(bool fwd, const void* in, void* out, size_t n_rows, size_t channels, size_t r, int dt,
                   void* stream) {
  if (dt != S2A_F32 && dt != S2A_BF16) return S2A_ERR_DTYPE;
  if (r == 0 || r > 0x7fffffffull || channels % r != 0) return S2A_ERR_SHAPE;
  if (n_rows * channels == 0) return S2A_OK;
  if (!in || !out) return S2A_ERR_NULL;
  if (misaligned(in, 16) || misaligned(out, 16)) return S2A_ERR_ALIGN;
  return launch_cap(fwd, dt, in, out, n_rows * (channels / r), (uint32_t)r, (cudaStream_t)stream) == cudaSuccess
             ? S2A_OK : S2A_ERR_CUDA;
}

int s2a_cap_fwd(const void* x, void* y, size_t n_rows, size_t channels, size_t r, int dt, void* cuda_stream) {
  return run_cap(true, x, y, n_rows, channels, r, dt, cuda_stream);
}

int s2a_cap_bwd(const void* grad_out, void* grad_in, size_t n_rows, size_t channels, size_t r, int dt,
                void* cuda_stream) {
  return run_cap(false, grad_out, grad_in, n_rows, channels, r, dt, cuda_stream);
}

int s2a_lrp_fwd(const void* x, const float* A, const float* B, void* y, size_t batch, size_t tokens,
                size_t channels, size_t rank, int dt, void* cuda_stream) {
  if (dt != S2A_F32 && dt != S2A_BF16) return S2A_ERR_DTYPE;
  if (batch > 0xffffffffull || tokens > 0xffffffffull || channels > 0xffffffffull || rank > 0xffffffffull)
    return S2A_ERR_SHAPE;
  if (batch * tokens * channels == 0) return S2A_OK;
  if (!x || !y || (rank > 0 && (!A || !B))) return S2A_ERR_NULL;
  if (misaligned(x, 16) || misaligned(y, 16) || misaligned(A, 4) || misaligned(B, 4)) return S2A_ERR_ALIGN;
  return launch_lrp_fwd(dt, x, A, B, y, (uint32_t)batch, (uint32_t)tokens, (uint32_t)channels, (uint32_t)rank,
                        (cudaStream_t)cuda_stream) == cudaSuccess ? S2A_OK : S2A_ERR_CUDA;
}

int s2a_silu_fwd(const void* x, void* y, uint8_t* codes, float* meta, size_t n_elems, size_t row_len, int dt,
                 void* cuda_stream) {
  return run(kSiluFwd, x, y, codes, meta, n_elems, row_len, dt, cuda_stream);
}

int s2a_silu_bwd(const void* grad_out, const uint8_t* codes, const float* meta, void* grad_in, size_t n_elems,
                 size_t row_len, int dt, void* cuda_stream) {
  return run(kSiluBwd, grad_out, grad_in, const_cast<uint8_t*>(codes), const_cast<float*>(meta), n_elems, row_len,
             dt, cuda_stream);
}

size_t s2a_tensor_range_scratch_bytes(size_t n_elems) { return (size_t)tensor_range_scratch_bytes(n_elems); }

int s2a_gelu_fwd_tensor_range(const void* x, void* y, uint8_t* codes, float* meta, void* scratch,
                              size_t n_elems, size_t row_len, int dt, void* cuda_stream) {
  int rc = check_args(x, y, codes, meta, n_elems, row_len, dt);
  if (rc != S2A_OK || n_elems == 0) return rc;
  if (!scratch) return S2A_ERR_NULL;
  if (misaligned(scratch, 8)) return S2A_ERR_ALIGN;
  return launch_gelu_fwd_tensor_range(dt, x, y, codes, meta, (float*)scratch, n_elems, n_elems / row_len,
                                      (cudaStream_t)cuda_stream) == cudaSuccess ? S2A_OK : S2A_ERR_CUDA;
}

size_t s2a_tensor_range_static_max_elems(void) { return (size_t)tensor_range_static_max_elems(); }

int s2a_gelu_fwd_tensor_range_static(const void* x, void* y, uint8_t* codes, float* meta, size_t n_elems,
                                     size_t row_len, int dt, void* cuda_stream) {
  int rc = check_args(x, y, codes, meta, n_elems, row_len, dt);
  if (rc != S2A_OK || n_elems == 0) return rc;
  if (n_elems > tensor_range_static_max_elems()) return S2A_ERR_TOO_LARGE;
  return launch_gelu_fwd_tensor_range_static(dt, x, y, codes, meta, n_elems, n_elems / row_len,
                                             (cudaStream_t)cuda_stream) == cudaSuccess ? S2A_OK : S2A_ERR_CUDA;
}

size_t s2a_mask_bytes(size_t n_elems) { return (n_elems + 7) / 8; }

static int run_relu(bool fwd, const void* in, void* out, uint8_t* mask, size_t n, int dt, void* stream) {
  if (dt != S2A_F32 && dt != S2A_BF16) return S2A_ERR_DTYPE;
  if (n == 0) return S2A_OK;
  if (!in || !out || !mask) return S2A_ERR_NULL;
  if (misaligned(in, 16) || misaligned(out, 16)) return S2A_ERR_ALIGN;
  return launch_relu(fwd, dt, in, out, mask, n, (cudaStream_t)stream) == cudaSuccess ? S2A_OK : S2A_ERR_CUDA;
}

int s2a_relu_fwd(const void* x, void* y, uint8_t* mask, size_t n_elems, int dt, void* cuda_stream) {
  return run_relu(true, x, y, mask, n_elems, dt, cuda_stream);
}

int s2a_relu_bwd(const void* grad_out, const uint8_t* mask, void* grad_in, size_t n_elems, int dt,
                 void* cuda_stream) {
  return run_relu(false, grad_out, grad_in, const_cast<uint8_t*>(mask), n_elems, dt, cuda_stream);
}

size_t s2a_codes_bytes_bits(size_t n_elems, int bits) {
  return (bits == 2 || bits == 4 || bits == 8) ? (n_elems * (size_t)bits + 7) / 8 : 0;
}

// General code width: 4 goes to the ordinary entry points.  At 2 and 8 bits the GELU
// kernels have a pipelined form for rows of whole 16-byte vectors; everything else, and
// the rows left over, run row at a time.
static int run_bits(int kernel, const void* in, void* out, uint8_t* codes, float* meta, size_t n, size_t row_len,
                    int bits, int dt, void* stream) {
  if (bits == 4) return run(kernel, in, out, codes, meta, n, row_len, dt, stream);
  if (bits != 2 && bits != 8) return S2A_ERR_SHAPE;
  int rc = check_args(in, out, codes, meta, n, row_len, dt);
  if (rc != S2A_OK || n == 0) return rc;
  cudaStream_t st = (cudaStream_t)stream;
  const uint64_t n_rows = n / row_len;
  uint64_t done_rows = 0;
  TilePlan p = plan_tile(kernel, dt, n_rows, (uint32_t)row_len, bits);
  if (p.tile_rows != 0 && p.n_tiles != 0 && !misaligned(meta, 16)) {
    TileArgs ta{in, out, codes, meta, (uint32_t)row_len, p.n_tiles};
    if (launch_tile(kernel, dt, p, ta, st) != cudaSuccess) return S2A_ERR_CUDA;
    done_rows = p.n_tiles * p.tile_rows;
  }
  if (done_rows < n_rows) {
    RowwiseArgs ra{in, out, codes, meta, done_rows, n_rows - done_rows, (uint32_t)row_len};
    if (launch_rowwise(kernel, dt, ra, st, bits) != cudaSuccess) return S2A_ERR_CUDA;
  }
  return S2A_OK;
}

int s2a_gelu_fwd_bits(const void* x, void* y, uint8_t* codes, float* meta, size_t n_elems, size_t row_len,
                      int bits, int dt, void* cuda_stream) {
  return run_bits(kGeluFwd, x, y, codes, meta, n_elems, row_len, bits, dt, cuda_stream);
}
int s2a_gelu_bwd_bits(const void* grad_out, const uint8_t* codes, const float* meta, void* grad_in, size_t n_elems,
                      size_t row_len, int bits, int dt, void* cuda_stream) {
  return run_bits(kGeluBwd, grad_out, grad_in, const_cast<uint8_t*>(codes), const_cast<float*>(meta), n_elems,
                  row_len, bits, dt, cuda_stream);
}
int s2a_softmax_fwd_bits(const void* x, void* y, uint8_t* codes, float* meta, size_t n_elems, size_t row_len,
                         int bits, int dt, void* cuda_stream) {
  return run_bits(kSoftmaxFwd, x, y, codes, meta, n_elems, row_len, bits, dt, cuda_stream);
}
int s2a_softmax_bwd_bits(const void* grad_out, const uint8_t* codes, const float* meta, void* grad_in,
                         size_t n_elems, size_t row_len, int bits, int dt, void* cuda_stream) {
  return run_bits(kSoftmaxBwd, grad_out, grad_in, const_cast<uint8_t*>(codes), const_cast<float*>(meta), n_elems,
                  row_len, bits, dt, cuda_stream);
}

// ---- layer norm, dropout, relative position bias

static size_t elem_bytes(int dt) { return dt == S2A_F32 ? 4 : 2; }

// Whether n_rows rows of row_bytes, row_stride bytes apart, reach into another such set (in place, with equal rows, is
// asked separately).  Two sets of one stride may interleave: slices of one buffer side by side.
static bool rows_overlap(const void* a, size_t a_stride, const void* b, size_t b_stride, size_t n_rows, size_t row_bytes) {
  const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
  const uintptr_t span_a = (n_rows - 1) * a_stride + row_bytes, span_b = (n_rows - 1) * b_stride + row_bytes;
  if (pa + span_a <= pb || pb + span_b <= pa) return false;
  if (a_stride == b_stride && n_rows > 1 && a_stride >= row_bytes) {
    const uintptr_t d = pa < pb ? (pb - pa) % a_stride : (pa - pb) % a_stride;
    return d < row_bytes || a_stride - d < row_bytes;
  }
  return true;
}

// The layout rules of one output of a row-wise call against one of its inputs: the same rows, or apart.
static bool bad_rows(const void* in, size_t in_stride, const void* out, size_t out_stride, size_t n_rows, size_t row_bytes) {
  if (in == out && (in_stride == out_stride || n_rows == 1)) return false;
  return rows_overlap(in, in_stride, out, out_stride, n_rows, row_bytes);
}

static bool bytes_overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  return (uintptr_t)a < (uintptr_t)b + b_bytes && (uintptr_t)b < (uintptr_t)a + a_bytes;
}

// n_rows rows of row_len elements, `stride` apart, must be addressable.
static bool bad_stride(size_t n_rows, size_t row_len, size_t stride) {
  return n_rows > 1 && stride != 0 && (n_rows - 1) > (((size_t)1 << 60) - row_len) / stride;
}

size_t s2a_layernorm_scratch_bytes(size_t n_rows, size_t row_len) {
  return row_len == 0 || row_len > 0x7fffffffull ? 0 : (size_t)layernorm_scratch_bytes(n_rows, (uint32_t)row_len);
}

int s2a_layernorm_fwd(const void* x, const void* gamma, const void* beta, void* y, float* stats, size_t n_rows,
                      size_t row_len, size_t x_stride, size_t y_stride, float eps, int dt, int wdt, void* cuda_stream) {
  if ((dt != S2A_F32 && dt != S2A_BF16) || (wdt != S2A_F32 && wdt != S2A_BF16)) return S2A_ERR_DTYPE;
  if (row_len == 0 || row_len > 0x7fffffffull || (n_rows > 1 && y_stride < row_len) ||
      bad_stride(n_rows, row_len, x_stride) || bad_stride(n_rows, row_len, y_stride))
    return S2A_ERR_SHAPE;
  if (!(eps >= 0.0f) || eps > 3.4028234e38f) return S2A_ERR_VALUE;
  if (n_rows == 0) return S2A_OK;
  if (!x || !y) return S2A_ERR_NULL;
  const size_t es = elem_bytes(dt);
  if (misaligned(x, es) || misaligned(y, es) || misaligned(gamma, elem_bytes(wdt)) || misaligned(beta, elem_bytes(wdt)) ||
      misaligned(stats, 8))
    return S2A_ERR_ALIGN;
  if (bad_rows(x, x_stride * es, y, y_stride * es, n_rows, row_len * es)) return S2A_ERR_OVERLAP;
  return launch_layernorm_fwd(dt, wdt, x, gamma, beta, y, stats, n_rows, (uint32_t)row_len, x_stride, y_stride, eps,
                              (cudaStream_t)cuda_stream) == cudaSuccess ? S2A_OK : S2A_ERR_CUDA;
}

int s2a_layernorm_bwd(const void* grad_out, const void* x, const void* gamma, const float* stats, void* grad_in,
                      void* grad_gamma, void* grad_beta, void* scratch, size_t n_rows, size_t row_len,
                      size_t grad_out_stride, size_t x_stride, size_t grad_in_stride, int dt, int wdt, void* cuda_stream) {
  if ((dt != S2A_F32 && dt != S2A_BF16) || (wdt != S2A_F32 && wdt != S2A_BF16)) return S2A_ERR_DTYPE;
  if (row_len == 0 || row_len > 0x7fffffffull || (n_rows > 1 && grad_in_stride < row_len) ||
      bad_stride(n_rows, row_len, x_stride) || bad_stride(n_rows, row_len, grad_out_stride) ||
      bad_stride(n_rows, row_len, grad_in_stride))
    return S2A_ERR_SHAPE;
  const bool sums = grad_gamma || grad_beta;
  if (n_rows > 0 && (!grad_out || !x || !stats || !grad_in || (sums && !scratch))) return S2A_ERR_NULL;
  const size_t es = elem_bytes(dt), ws = elem_bytes(wdt);
  if (misaligned(grad_out, es) || misaligned(x, es) || misaligned(grad_in, es) || misaligned(stats, 8) ||
      misaligned(gamma, ws) || misaligned(grad_gamma, ws) || misaligned(grad_beta, ws) || misaligned(scratch, 16))
    return S2A_ERR_ALIGN;
  if (n_rows > 0 && (bad_rows(grad_out, grad_out_stride * es, grad_in, grad_in_stride * es, n_rows, row_len * es) ||
                     bad_rows(x, x_stride * es, grad_in, grad_in_stride * es, n_rows, row_len * es)))
    return S2A_ERR_OVERLAP;
  return launch_layernorm_bwd(dt, wdt, grad_out, x, gamma, stats, grad_in, grad_gamma, grad_beta, (float*)scratch, n_rows,
                              (uint32_t)row_len, grad_out_stride, x_stride, grad_in_stride, (cudaStream_t)cuda_stream) ==
                 cudaSuccess ? S2A_OK : S2A_ERR_CUDA;
}

static int run_dropout(const void* x, const void* residual, void* y, size_t n, const uint64_t* rng, uint64_t site, double p,
                       int dt, void* stream) {
  if (dt != S2A_F32 && dt != S2A_BF16) return S2A_ERR_DTYPE;
  if (!(p >= 0.0 && p <= 1.0)) return S2A_ERR_VALUE;
  if (n > ((size_t)1 << 60)) return S2A_ERR_SHAPE;
  if (n == 0) return S2A_OK;
  if (!x || !y || !rng) return S2A_ERR_NULL;
  if (misaligned(x, 16) || misaligned(residual, 16) || misaligned(y, 16) || misaligned(rng, 8)) return S2A_ERR_ALIGN;
  const size_t bytes = n * elem_bytes(dt);
  if ((x != y && bytes_overlap(x, bytes, y, bytes)) || (residual && residual != y && bytes_overlap(residual, bytes, y, bytes)))
    return S2A_ERR_OVERLAP;
  return launch_dropout(dt, x, residual, y, n, rng, site, s2a_dropout_threshold(p), (cudaStream_t)stream) == cudaSuccess
             ? S2A_OK : S2A_ERR_CUDA;
}

uint32_t s2a_dropout_threshold(double p) { return !(p > 0.0) ? 0u : (p >= 1.0 ? 65536u : (uint32_t)nearbyint(65536.0 * p)); }

int s2a_dropout_fwd(const void* x, const void* residual, void* y, size_t n_elems, const uint64_t* rng, uint64_t site,
                    double p, int dt, void* cuda_stream) {
  return run_dropout(x, residual, y, n_elems, rng, site, p, dt, cuda_stream);
}

int s2a_dropout_bwd(const void* grad_out, void* grad_in, size_t n_elems, const uint64_t* rng, uint64_t site, double p, int dt,
                    void* cuda_stream) {
  return run_dropout(grad_out, nullptr, grad_in, n_elems, rng, site, p, dt, cuda_stream);
}

static bool bad_bias_shape(size_t batch, size_t heads, size_t tq, size_t tk, size_t n_buckets) {
  if (batch > 0x7fffffffull || heads == 0 || heads > 65535u || tq > 0x7fffffffull || tk > 0x7fffffffull || n_buckets == 0 ||
      n_buckets > kMaxBuckets)
    return true;
  const size_t slab = tq * tk;
  return slab > ((size_t)1 << 36) || (slab != 0 && batch * heads > ((size_t)1 << 60) / slab);
}

size_t s2a_relbias_scratch_bytes(size_t batch, size_t heads, size_t tq, size_t tk, size_t n_buckets) {
  if (bad_bias_shape(batch, heads, tq, tk, n_buckets) || batch * tq * tk == 0) return 0;
  return (size_t)relbias_scratch_bytes((uint32_t)heads, (uint32_t)n_buckets);
}

int s2a_relbias_fwd(const void* x, const void* table, const int32_t* buckets, int by_distance, void* y, size_t batch,
                    size_t heads, size_t tq, size_t tk, size_t n_buckets, int dt, int wdt, void* cuda_stream) {
  if ((dt != S2A_F32 && dt != S2A_BF16) || (wdt != S2A_F32 && wdt != S2A_BF16)) return S2A_ERR_DTYPE;
  if (bad_bias_shape(batch, heads, tq, tk, n_buckets)) return S2A_ERR_SHAPE;
  if (batch * tq * tk == 0) return S2A_OK;
  if (!x || !table || !buckets || !y) return S2A_ERR_NULL;
  if (misaligned(x, 16) || misaligned(y, 16) || misaligned(table, elem_bytes(wdt)) || misaligned(buckets, 4))
    return S2A_ERR_ALIGN;
  const size_t bytes = batch * heads * tq * tk * elem_bytes(dt);
  if (x != y && bytes_overlap(x, bytes, y, bytes)) return S2A_ERR_OVERLAP;
  return launch_relbias_fwd(dt, wdt, x, table, buckets, by_distance != 0, y, (uint32_t)batch, (uint32_t)heads, (uint32_t)tq,
                            (uint32_t)tk, (uint32_t)n_buckets, (cudaStream_t)cuda_stream) == cudaSuccess
             ? S2A_OK : S2A_ERR_CUDA;
}

int s2a_relbias_bwd(const void* grad_out, const int32_t* buckets, int by_distance, void* grad_table, void* scratch,
                    size_t batch, size_t heads, size_t tq, size_t tk, size_t n_buckets, int dt, int wdt, void* cuda_stream) {
  if ((dt != S2A_F32 && dt != S2A_BF16) || (wdt != S2A_F32 && wdt != S2A_BF16)) return S2A_ERR_DTYPE;
  if (bad_bias_shape(batch, heads, tq, tk, n_buckets)) return S2A_ERR_SHAPE;
  const bool empty = batch * tq * tk == 0;
  if (!grad_table || (!empty && (!grad_out || !buckets || !scratch))) return S2A_ERR_NULL;
  if (misaligned(grad_out, 16) || misaligned(buckets, 4) || misaligned(grad_table, elem_bytes(wdt)) || misaligned(scratch, 16))
    return S2A_ERR_ALIGN;
  return launch_relbias_bwd(dt, wdt, grad_out, buckets, by_distance != 0, grad_table, (float*)scratch, (uint32_t)batch,
                            (uint32_t)heads, (uint32_t)tq, (uint32_t)tk, (uint32_t)n_buckets, (cudaStream_t)cuda_stream) ==
                 cudaSuccess ? S2A_OK : S2A_ERR_CUDA;
}

int s2a_relbias_log_buckets(int32_t* buckets, int64_t first_distance, size_t count, size_t n_buckets, size_t max_distance,
                            int bidirectional) {
  const size_t side = bidirectional ? n_buckets / 2 : n_buckets;
  if (n_buckets > kMaxBuckets || side < 2 || (bidirectional && n_buckets % 2 != 0)) return S2A_ERR_SHAPE;
  if (max_distance <= side / 2 || max_distance > 0x7fffffffull || count > ((size_t)1 << 40) ||
      first_distance < -((int64_t)1 << 40) || first_distance > ((int64_t)1 << 40))
    return S2A_ERR_VALUE;
  if (count == 0) return S2A_OK;
  if (!buckets) return S2A_ERR_NULL;
  if (misaligned(buckets, 4)) return S2A_ERR_ALIGN;
  log_buckets(buckets, first_distance, count, (uint32_t)n_buckets, (uint32_t)max_distance, bidirectional != 0);
  return S2A_OK;
}

int s2a_device_error(unsigned int* flags, int clear) {
  if (!flags) return S2A_ERR_NULL;
  return read_error_word(flags, clear != 0) == cudaSuccess ? S2A_OK : S2A_ERR_CUDA;
}

int s2a_selftest_wait_expiry(void* cuda_stream) {
  return launch_wait_expiry_probe((cudaStream_t)cuda_stream) == cudaSuccess ? S2A_OK : S2A_ERR_CUDA;
}

int s2a_selftest_exp2_monotone(unsigned long long* out_of_order, void* cuda_stream) {
  if (!out_of_order) return S2A_ERR_NULL;
  return count_exp2_out_of_order(out_of_order, (cudaStream_t)cuda_stream) == cudaSuccess ? S2A_OK : S2A_ERR_CUDA;
}

int s2a_describe_plan(int kernel, size_t n_elems, size_t row_len, int dt, char* out, size_t cap) {
  if (!out || cap == 0) return S2A_ERR_NULL;
  out[0] = 0;
  if (kernel < 0 || kernel > 5) return S2A_ERR_SHAPE;
  if (dt != S2A_F32 && dt != S2A_BF16) return S2A_ERR_DTYPE;
  if (row_len == 0 || row_len > 0x7fffffffull || n_elems % row_len != 0) return S2A_ERR_SHAPE;
  const uint64_t n_rows = n_elems / row_len;
  TilePlan p = plan_tile(kernel, dt, n_rows, (uint32_t)row_len);
  if (p.tile_rows == 0 || p.n_tiles == 0) {
    snprintf(out, cap, "rowwise rows=%llu", (unsigned long long)n_rows);
  } else {
    snprintf(out, cap,
             "tile variant=%s rows/tile=%u unit=%u vec=%u iters=%u warps=%u stages=%u smem=%u grid=%u "
             "group=%u spread=%u ragged_codes=%u tiles=%llu tail_rows=%llu",
             p.variant == kVariantStream ? "stream" : (p.variant == kVariantPairFixed ? "pair-fixed" : (p.variant == kVariantAny ? "any-length" : "generic")),
             p.tile_rows, p.unit_lanes, p.vec_elems, p.iters, p.warps, p.stages, p.smem_bytes,
             p.grid, p.rows_per_group, p.spread_units, p.ragged_codes, (unsigned long long)p.n_tiles,
             (unsigned long long)(n_rows - p.n_tiles * p.tile_rows));
  }
  return S2A_OK;
}

}  // extern "C"
