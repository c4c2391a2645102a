// C ABI of the 4-bit float operators: argument checks and the sequence of launches.  See include/b2conv.h for the contract of each
// entry point.
#include "fp4_internal.h"

using namespace b2c;

namespace {

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool wide_type(int t) { return t == B2C_F32 || t == B2C_F16 || t == B2C_BF16; }
bool fp4_format(int f) { return f == B2C_MXFP4 || f == B2C_NVFP4; }

int from_cuda(cudaError_t e) {
  if (e == cudaSuccess) return B2C_OK;
  set_last_cuda_error((int)e);
  return B2C_E_CUDA;
}

// The workspace of an expert layer, in order; each part starts on a 256-byte boundary.
struct ExpertsLayout {
  size_t offsets, rows, sort, xq, xs, hq, hs, y, done, total;
};
int experts_layout(const b2c_fp4_experts_desc* d, int64_t tokens, ExpertsLayout* l) {
  if (!d || tokens < 0) return B2C_E_INVALID_ARG;
  if (d->hidden < 32 || d->inter < 32 || d->hidden % 32 || d->inter % 32) return B2C_E_INVALID_ARG;
  if (d->experts < 1 || d->topk < 1 || d->topk > d->experts || !wide_type(d->type) || !fp4_format(d->format)) return B2C_E_INVALID_ARG;
  if (d->experts > kMaxExperts || d->topk > kMaxTopk || (long long)d->hidden * d->inter >= kMaxStride) return B2C_E_UNSUPPORTED;
  if (d->hidden > kMaxCols || d->inter > kMaxCols) return B2C_E_UNSUPPORTED;
  if (tokens > kMaxRows / d->topk) return B2C_E_UNSUPPORTED;
  const size_t pairs = (size_t)tokens * d->topk;
  size_t at = 0;
  auto part = [&](size_t bytes) {
    const size_t here = at;
    at = (at + bytes + 255) / 256 * 256;
    return here;
  };
  l->offsets = part(4 * ((size_t)d->experts + 1));
  l->rows = part(4 * pairs);
  l->sort = part(route_sort_workspace((long long)pairs, d->experts));
  l->xq = part(pairs * d->hidden / 2);
  l->xs = part(pairs * fp4_scale_pitch(d->hidden, d->format));
  l->hq = part(pairs * d->inter / 2);
  l->hs = part(pairs * fp4_scale_pitch(d->inter, d->format));
  l->y = part(pairs * d->hidden * 4);
  l->done = part(4 * (((size_t)d->hidden + kTileM - 1) / kTileM));
  l->total = at;
  return B2C_OK;
}

}  // namespace

extern "C" {

int b2c_fp4_quantize(const void* x, int x_type, int64_t rows, int32_t cols, int64_t ldx, int format, const float* global_scale, void* q,
                     int64_t ldq, void* scale, int64_t ld_scale, void* cuda_stream) {
  if (!wide_type(x_type) || !fp4_format(format) || (format == B2C_MXFP4 && global_scale)) return B2C_E_INVALID_ARG;
  if (rows < 0 || cols < 1 || ldx < cols || ldq < (cols + 1ll) / 2 || ld_scale < fp4_scales(cols, format)) return B2C_E_INVALID_ARG;
  if (rows == 0) return B2C_OK;
  if (!x || !q || !scale || !aligned(x, type_bytes(x_type)) || !aligned(global_scale, 4)) return B2C_E_INVALID_ARG;
  if (rows > kMaxRows || cols > kMaxCols) return B2C_E_UNSUPPORTED;
  Quantize4Args a = {};
  a.x = x;
  a.ldx = ldx;
  a.q = (uint8_t*)q;
  a.ldq = ldq;
  a.scale = (uint8_t*)scale;
  a.lds = ld_scale;
  a.global = global_scale;
  a.rows = rows;
  a.cols = cols;
  a.x_type = x_type;
  a.format = format;
  return from_cuda(launch_fp4_quantize(a, (cudaStream_t)cuda_stream));
}

int b2c_fp4_dequantize(const void* q, int64_t ldq, const void* scale, int64_t ld_scale, int64_t rows, int32_t cols, int format,
                       const float* global_scale, void* y, int y_type, int64_t ldy, void* cuda_stream) {
  if (!wide_type(y_type) || !fp4_format(format) || (format == B2C_MXFP4 && global_scale)) return B2C_E_INVALID_ARG;
  if (rows < 0 || cols < 1 || ldy < cols || ldq < (cols + 1ll) / 2 || ld_scale < fp4_scales(cols, format)) return B2C_E_INVALID_ARG;
  if (rows == 0) return B2C_OK;
  if (!y || !q || !scale || !aligned(y, type_bytes(y_type)) || !aligned(global_scale, 4)) return B2C_E_INVALID_ARG;
  if (rows > kMaxRows || cols > kMaxCols) return B2C_E_UNSUPPORTED;
  Dequantize4Args a = {};
  a.q = (const uint8_t*)q;
  a.ldq = ldq;
  a.scale = (const uint8_t*)scale;
  a.lds = ld_scale;
  a.global = global_scale;
  a.rows = rows;
  a.cols = cols;
  a.y = y;
  a.ldy = ldy;
  a.y_type = y_type;
  a.format = format;
  return from_cuda(launch_fp4_dequantize(a, (cudaStream_t)cuda_stream));
}

int b2c_fp4_matmul(const b2c_fp4_matmul_desc* d, int64_t rows, const void* a, int64_t lda, const void* a_scale, int64_t ld_a_scale, const void* b,
                   const void* b_scale, int64_t ld_b_scale, const float* alpha, const int32_t* offsets, void* y, int64_t ldy, void* cuda_stream) {
  if (!d || d->N < 1 || d->K < 32 || d->K % 32 || d->groups < 1 || rows < 0) return B2C_E_INVALID_ARG;
  if (!fp4_format(d->format) || !wide_type(d->y_type)) return B2C_E_INVALID_ARG;
  const long long scales = fp4_scales(d->K, d->format);
  if (lda < d->K / 2 || lda % 16 || ld_a_scale < scales || ld_a_scale % 16 || ld_b_scale < scales || ld_b_scale % 16 || ldy < d->N) return B2C_E_INVALID_ARG;
  if (d->groups > 1 && !offsets) return B2C_E_INVALID_ARG;
  if (d->groups > kMaxExperts || rows > kMaxRows || d->N > kMaxCols || d->K > kMaxCols) return B2C_E_UNSUPPORTED;
  // (strides that a tensor map can hold)
  if (lda >= kMaxStride || ld_a_scale >= kMaxStride || ld_b_scale >= kMaxStride / d->N || (long long)d->N * (d->K / 2) >= kMaxStride ||
      ldy >= kMaxStride / type_bytes(d->y_type))
    return B2C_E_UNSUPPORTED;
  if (rows == 0) return B2C_OK;
  if (!a || !a_scale || !b || !b_scale || !y) return B2C_E_INVALID_ARG;
  if (!aligned(a, 16) || !aligned(b, 16) || !aligned(a_scale, 16) || !aligned(b_scale, 16) || !aligned(alpha, 4) || !aligned(offsets, 4) ||
      !aligned(y, type_bytes(d->y_type)))
    return B2C_E_INVALID_ARG;
  Matmul4Args m = {};
  m.a = (const uint8_t*)a;
  m.lda = lda;
  m.a_scale = (const uint8_t*)a_scale;
  m.lds = ld_a_scale;
  m.b = (const uint8_t*)b;
  m.b_scale = (const uint8_t*)b_scale;
  m.ldbs = ld_b_scale;
  m.alpha = alpha;
  m.offsets = offsets;
  m.y = y;
  m.ldy = ldy;
  m.rows = (int)rows;
  m.N = d->N;
  m.K = d->K;
  m.groups = d->groups;
  m.format = d->format;
  m.y_type = d->y_type;
  return launch_fp4_matmul(m, (cudaStream_t)cuda_stream);
}

int b2c_fp4_experts_workspace_bytes(const b2c_fp4_experts_desc* d, int64_t tokens, size_t* bytes) {
  if (!bytes) return B2C_E_INVALID_ARG;
  ExpertsLayout l;
  const int rc = experts_layout(d, tokens, &l);
  if (rc == B2C_OK) *bytes = l.total;
  return rc;
}

int b2c_fp4_experts(const b2c_fp4_experts_desc* d, int64_t tokens, const void* x, int64_t ldx, const int32_t* ids, const float* weights, const void* w1,
                    const void* w1_scale, int64_t ld1, const void* w2, const void* w2_scale, int64_t ld2, const float* x_global, const float* w1_global,
                    const float* h_global, const float* w2_global, void* y, int64_t ldy, void* workspace, void* cuda_stream) {
  ExpertsLayout l;
  int rc = experts_layout(d, tokens, &l);
  if (rc != B2C_OK) return rc;
  if (d->format == B2C_MXFP4 && (x_global || w1_global || h_global || w2_global)) return B2C_E_INVALID_ARG;
  if (ldx < d->hidden || ldy < d->hidden) return B2C_E_INVALID_ARG;
  if (ld1 < fp4_scales(d->hidden, d->format) || ld1 % 16 || ld2 < fp4_scales(d->inter, d->format) || ld2 % 16) return B2C_E_INVALID_ARG;
  if (ld1 >= kMaxStride / d->inter || ld2 >= kMaxStride / d->hidden) return B2C_E_UNSUPPORTED;
  if (tokens == 0) return B2C_OK;
  if (!x || !ids || !weights || !w1 || !w1_scale || !w2 || !w2_scale || !y || !workspace) return B2C_E_INVALID_ARG;
  if (!aligned(x, type_bytes(d->type)) || !aligned(y, type_bytes(d->type)) || !aligned(ids, 4) || !aligned(weights, 4) || !aligned(w1, 16) ||
      !aligned(w2, 16) || !aligned(w1_scale, 16) || !aligned(w2_scale, 16) || !aligned(x_global, 4) || !aligned(w1_global, 4) || !aligned(h_global, 4) ||
      !aligned(w2_global, 4) || !aligned(workspace, 16))
    return B2C_E_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  char* ws = (char*)workspace;
  const long long pairs = tokens * d->topk;
  // Two kernels where an expert has few rows (its tiles are 16 rows wide, and are quantised again for every tile of columns): us by them and by
  // the five launches below, NV: 2048 x 1024, 4 of 64 experts: 1 token 14 and 20, 16 37 and 45, 64 58 and 58, 100 76 and 64 (MX 14 and 18, 36 and 42, 53
  // and 54, 67 and 60);  1024 x 512: 16 tokens 22 and 25, 64 32 and 31, 100 40 and 32;  4096 x 1024, 4 of 32: 16 51 and 56, 64 84 and 64.
  if (pairs <= kFewPairs && pairs <= 4ll * d->experts) {
    Few4Args f = {};
    f.x = x;
    f.ldx = ldx;
    f.ids = ids;
    f.weights = weights;
    f.w1 = (const uint8_t*)w1;
    f.w1_scale = (const uint8_t*)w1_scale;
    f.w2 = (const uint8_t*)w2;
    f.w2_scale = (const uint8_t*)w2_scale;
    f.ld1 = ld1;
    f.ld2 = ld2;
    f.x_global = x_global;
    f.w1_global = w1_global;
    f.h_global = h_global;
    f.w2_global = w2_global;
    f.hq = (uint8_t*)(ws + l.hq);
    f.hs = (uint8_t*)(ws + l.hs);
    f.ldhs = fp4_scale_pitch(d->inter, d->format);
    f.part = (float*)(ws + l.y);
    f.done = (int32_t*)(ws + l.done);
    f.y = y;
    f.ldy = ldy;
    f.pairs = (int)pairs;
    f.topk = d->topk;
    f.experts = d->experts;
    f.hidden = d->hidden;
    f.inter = d->inter;
    f.type = d->type;
    f.format = d->format;
    return launch_fp4_few_experts(f, st);
  }
  int32_t* offsets = (int32_t*)(ws + l.offsets);
  int32_t* rows = (int32_t*)(ws + l.rows);
  rc = from_cuda(launch_route_sort(ids, pairs, d->experts, offsets, rows, nullptr, (int32_t*)(ws + l.sort), st));
  if (rc != B2C_OK) return rc;
  Quantize4Args q = {};
  q.x = x;
  q.ldx = ldx;
  q.q = (uint8_t*)(ws + l.xq);
  q.ldq = d->hidden / 2;
  q.scale = (uint8_t*)(ws + l.xs);
  q.lds = fp4_scale_pitch(d->hidden, d->format);
  q.global = x_global;
  q.rows = tokens;
  q.cols = d->hidden;
  q.x_type = d->type;
  q.format = d->format;
  q.map = rows;
  q.copies = d->topk;
  rc = from_cuda(launch_fp4_quantize(q, st));
  if (rc != B2C_OK) return rc;

  Matmul4Args m = {};
  m.a = q.q;
  m.lda = q.ldq;
  m.a_scale = q.scale;
  m.lds = q.lds;
  m.b = (const uint8_t*)w1;
  m.b_scale = (const uint8_t*)w1_scale;
  m.ldbs = ld1;
  m.alpha = w1_global;
  m.alpha2 = x_global;
  m.offsets = offsets;
  m.y = ws + l.hq;
  m.ldy = d->inter / 2;
  m.y_scale = (uint8_t*)(ws + l.hs);
  m.ldys = fp4_scale_pitch(d->inter, d->format);
  m.y_global = h_global;
  m.rows = (int)pairs;
  m.N = d->inter;
  m.K = d->hidden;
  m.groups = d->experts;
  m.format = d->format;
  m.gated = 1;
  rc = launch_fp4_matmul(m, st);
  if (rc != B2C_OK) return rc;

  m.a = (const uint8_t*)m.y;
  m.lda = m.ldy;
  m.a_scale = m.y_scale;
  m.lds = m.ldys;
  m.b = (const uint8_t*)w2;
  m.b_scale = (const uint8_t*)w2_scale;
  m.ldbs = ld2;
  m.alpha = w2_global;
  m.alpha2 = h_global;
  m.y = ws + l.y;
  m.ldy = d->hidden;
  m.y_scale = nullptr;
  m.ldys = 0;
  m.y_global = nullptr;
  m.N = d->hidden;
  m.K = d->inter;
  m.y_type = B2C_F32;  // (a slot's row is a partial sum: y is rounded once)
  m.gated = 0;
  m.early = 1;  // (the first product read its offsets after the sort had ended, and lets no later kernel start before that)
  rc = launch_fp4_matmul(m, st);
  if (rc != B2C_OK) return rc;
  return from_cuda(launch_route_combine(m.y, B2C_F32, pairs, m.ldy, rows, weights, tokens, d->topk, d->hidden, y, d->type, ldy, st));
}

int b2c_fp4_status(int32_t* status) {
  if (!status) return B2C_E_INVALID_ARG;
  return fp4_status_read_and_clear(status);
}

int b2c_selftest_fp4_wait(int form, void* cuda_stream) {
  if (form < 0 || form > 2) return B2C_E_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  return from_cuda(form == 0 ? fp4_rows_wait_selftest(st) : (form == 1 ? fp4_pair_wait_selftest(st) : fp4_few_wait_selftest(st)));
}

}  // extern "C"
