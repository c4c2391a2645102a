// C ABI of the 8-bit float operators: argument checks and the sequence of launches.  See include/b2conv.h for the
// contract of each entry point.
#include "fp8_internal.h"

using namespace b2c;

namespace {

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool wide_type(int t) { return t == B2C_F32 || t == B2C_F16 || t == B2C_BF16; }
bool fp8_type(int t) { return t == B2C_E4M3 || t == B2C_E5M2; }

int from_cuda(cudaError_t e) {
  if (e == cudaSuccess) return B2C_OK;
  set_last_cuda_error((int)e);
  return B2C_E_CUDA;
}

int check_route(const b2c_route_desc& d) {
  if (d.experts < 1 || d.topk < 1 || d.groups < 1 || d.topk_groups < 1 || d.topk_groups > d.groups) return B2C_E_INVALID_ARG;
  if (d.experts % d.groups != 0 || (long long)d.topk > (long long)(d.experts / d.groups) * d.topk_groups) return B2C_E_INVALID_ARG;
  if (d.score != B2C_SCORE_SOFTMAX && d.score != B2C_SCORE_SIGMOID) return B2C_E_INVALID_ARG;
  if (d.group_score != B2C_GROUP_MAX && d.group_score != B2C_GROUP_TOP2) return B2C_E_INVALID_ARG;
  if ((d.renormalise != 0 && d.renormalise != 1) || !wide_type(d.logit_type)) return B2C_E_INVALID_ARG;
  if (d.experts > kMaxExperts || d.topk > kMaxTopk || d.groups > kMaxRouteGroups) return B2C_E_UNSUPPORTED;
  return B2C_OK;
}

// The workspace of an expert layer, in order; each part starts on a 256-byte boundary.
struct ExpertsLayout {
  size_t offsets, rows, sort, xq, xs, hq, hs, y, total;
};
int experts_layout(const b2c_experts_desc* d, int64_t tokens, ExpertsLayout* l) {
  if (!d || tokens < 0) return B2C_E_INVALID_ARG;
  if (d->hidden < 16 || d->inter < 16 || d->hidden % 16 || d->inter % 16) return B2C_E_INVALID_ARG;
  if (d->experts < 1 || d->topk < 1 || d->topk > d->experts || !wide_type(d->type)) return B2C_E_INVALID_ARG;
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
  l->xq = part(pairs * d->hidden);
  l->xs = part(4 * pairs * blocks_of(d->hidden));
  l->hq = part(pairs * d->inter);
  l->hs = part(4 * pairs * blocks_of(d->inter));
  l->y = part(pairs * d->hidden * 4);
  l->total = at;
  return B2C_OK;
}

}  // namespace

extern "C" {

int b2c_fp8_quantize(const void* x, int x_type, int64_t rows, int32_t cols, int64_t ldx, int block_rows, int q_type, void* q,
                     int64_t ldq, float* scale, int64_t ld_scale, void* cuda_stream) {
  if (!wide_type(x_type) || !fp8_type(q_type) || (block_rows != 1 && block_rows != kBlock)) return B2C_E_INVALID_ARG;
  if (rows < 0 || cols < 1 || ldx < cols || ldq < cols || ld_scale < blocks_of(cols)) return B2C_E_INVALID_ARG;
  if (rows == 0) return B2C_OK;
  if (!x || !q || !scale || !aligned(x, type_bytes(x_type)) || !aligned(scale, 4)) return B2C_E_INVALID_ARG;
  if (rows > kMaxRows || cols > kMaxCols) return B2C_E_UNSUPPORTED;
  QuantizeArgs a = {};
  a.x = x;
  a.ldx = ldx;
  a.q = (uint8_t*)q;
  a.ldq = ldq;
  a.scale = scale;
  a.lds = ld_scale;
  a.rows = rows;
  a.cols = cols;
  a.block_rows = block_rows;
  a.x_type = x_type;
  a.q_type = q_type;
  return from_cuda(launch_fp8_quantize(a, (cudaStream_t)cuda_stream));
}

int b2c_fp8_matmul(const b2c_matmul_desc* d, int64_t rows, const void* a, int64_t lda, const float* a_scale, int64_t ld_a_scale,
                   const void* b, const float* b_scale, const int32_t* offsets, void* y, int64_t ldy, void* cuda_stream) {
  if (!d || d->N < 1 || d->K < 16 || d->K % 16 || d->groups < 1 || rows < 0) return B2C_E_INVALID_ARG;
  if (!fp8_type(d->a_type) || !fp8_type(d->b_type) || !wide_type(d->y_type)) return B2C_E_INVALID_ARG;
  if (lda < d->K || lda % 16 || ld_a_scale < blocks_of(d->K) || ldy < d->N) return B2C_E_INVALID_ARG;
  if (d->groups > 1 && !offsets) return B2C_E_INVALID_ARG;
  if (d->groups > kMaxExperts || rows > kMaxRows || d->N > kMaxCols || d->K > kMaxCols) return B2C_E_UNSUPPORTED;
  // (strides that a tensor map can hold)
  if (lda >= kMaxStride || (long long)d->N * d->K >= kMaxStride || ldy * type_bytes(d->y_type) >= kMaxStride) return B2C_E_UNSUPPORTED;
  if (rows == 0) return B2C_OK;
  if (!a || !a_scale || !b || !b_scale || !y) return B2C_E_INVALID_ARG;
  if (!aligned(a, 16) || !aligned(b, 16) || !aligned(a_scale, 4) || !aligned(b_scale, 4) || !aligned(offsets, 4) ||
      !aligned(y, type_bytes(d->y_type)))
    return B2C_E_INVALID_ARG;
  MatmulArgs m = {};
  m.a = a;
  m.lda = lda;
  m.a_scale = a_scale;
  m.lds = ld_a_scale;
  m.b = b;
  m.b_scale = b_scale;
  m.offsets = offsets;
  m.y = y;
  m.ldy = ldy;
  m.rows = (int)rows;
  m.N = d->N;
  m.K = d->K;
  m.groups = d->groups;
  m.a_type = d->a_type;
  m.b_type = d->b_type;
  m.y_type = d->y_type;
  return launch_fp8_matmul(m, (cudaStream_t)cuda_stream);
}

int b2c_route(const b2c_route_desc* d, int64_t tokens, const void* logits, int64_t ld, const float* bias, float* weights,
              int32_t* ids, void* cuda_stream) {
  if (!d || tokens < 0) return B2C_E_INVALID_ARG;
  const int rc = check_route(*d);
  if (rc != B2C_OK) return rc;
  if (ld < d->experts) return B2C_E_INVALID_ARG;
  if (tokens > kMaxRows) return B2C_E_UNSUPPORTED;
  if (tokens == 0) return B2C_OK;
  if (!logits || !weights || !ids || !aligned(logits, type_bytes(d->logit_type)) || !aligned(bias, 4) || !aligned(weights, 4) ||
      !aligned(ids, 4))
    return B2C_E_INVALID_ARG;
  RouteArgs a = {*d, tokens, logits, ld, bias, weights, ids};
  return from_cuda(launch_route(a, (cudaStream_t)cuda_stream));
}

int b2c_route_sort_workspace_bytes(int64_t pairs, int32_t experts, size_t* bytes) {
  if (!bytes || pairs < 0 || experts < 1) return B2C_E_INVALID_ARG;
  if (pairs > kMaxRows || experts > kMaxExperts) return B2C_E_UNSUPPORTED;
  *bytes = route_sort_workspace(pairs, experts);
  return B2C_OK;
}

int b2c_route_sort(const int32_t* ids, int64_t pairs, int32_t experts, int32_t* offsets, int32_t* rows, int32_t* order,
                   void* workspace, void* cuda_stream) {
  if (pairs < 0 || experts < 1 || !offsets || !aligned(offsets, 4)) return B2C_E_INVALID_ARG;
  if (pairs > kMaxRows || experts > kMaxExperts) return B2C_E_UNSUPPORTED;
  if (pairs > 0 && (!ids || !rows || !aligned(ids, 4) || !aligned(rows, 4) || !aligned(order, 4))) return B2C_E_INVALID_ARG;
  if (!aligned(workspace, 16) || (route_sort_workspace(pairs, experts) > 0 && !workspace)) return B2C_E_INVALID_ARG;
  return from_cuda(launch_route_sort(ids, pairs, experts, offsets, rows, order, (int32_t*)workspace, (cudaStream_t)cuda_stream));
}

int b2c_route_combine(const void* y, int y_type, int64_t y_rows, int64_t ldy, const int32_t* rows, const float* weights, int64_t tokens,
                      int32_t topk, int32_t cols, void* out, int out_type, int64_t ldo, void* cuda_stream) {
  if (!wide_type(y_type) || !wide_type(out_type) || tokens < 0 || y_rows < 0 || topk < 1 || cols < 1 || ldy < cols || ldo < cols)
    return B2C_E_INVALID_ARG;
  if (topk > kMaxTopk || tokens > kMaxRows || cols > kMaxCols) return B2C_E_UNSUPPORTED;
  if (tokens == 0) return B2C_OK;
  if ((!y && y_rows > 0) || !rows || !weights || !out || !aligned(y, type_bytes(y_type)) || !aligned(rows, 4) || !aligned(weights, 4) ||
      !aligned(out, type_bytes(out_type)))
    return B2C_E_INVALID_ARG;
  return from_cuda(launch_route_combine(y, y_type, y_rows, ldy, rows, weights, tokens, topk, cols, out, out_type, ldo, (cudaStream_t)cuda_stream));
}

int b2c_experts_workspace_bytes(const b2c_experts_desc* d, int64_t tokens, size_t* bytes) {
  if (!bytes) return B2C_E_INVALID_ARG;
  ExpertsLayout l;
  const int rc = experts_layout(d, tokens, &l);
  if (rc == B2C_OK) *bytes = l.total;
  return rc;
}

int b2c_fp8_experts(const b2c_experts_desc* d, int64_t tokens, const void* x, int64_t ldx, const int32_t* ids, const float* weights,
                    const void* w1, const float* w1_scale, const void* w2, const float* w2_scale, void* y, int64_t ldy,
                    void* workspace, void* cuda_stream) {
  ExpertsLayout l;
  int rc = experts_layout(d, tokens, &l);
  if (rc != B2C_OK) return rc;
  if (ldx < d->hidden || ldy < d->hidden) return B2C_E_INVALID_ARG;
  if (tokens == 0) return B2C_OK;
  if (!x || !ids || !weights || !w1 || !w1_scale || !w2 || !w2_scale || !y || !workspace) return B2C_E_INVALID_ARG;
  if (!aligned(x, type_bytes(d->type)) || !aligned(y, type_bytes(d->type)) || !aligned(ids, 4) || !aligned(weights, 4) ||
      !aligned(w1, 16) || !aligned(w2, 16) || !aligned(w1_scale, 4) || !aligned(w2_scale, 4) || !aligned(workspace, 16))
    return B2C_E_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  char* ws = (char*)workspace;
  const long long pairs = tokens * d->topk;
  int32_t* offsets = (int32_t*)(ws + l.offsets);
  int32_t* rows = (int32_t*)(ws + l.rows);
  QuantizeArgs q = {};
  q.x = x;
  q.ldx = ldx;
  q.q = (uint8_t*)(ws + l.xq);
  q.ldq = d->hidden;
  q.scale = (float*)(ws + l.xs);
  q.lds = blocks_of(d->hidden);
  q.rows = tokens;
  q.cols = d->hidden;
  q.block_rows = 1;
  q.x_type = d->type;
  q.q_type = B2C_E4M3;
  q.map = rows;
  q.copies = d->topk;
  if (pairs <= kSmallPairs) {
    rc = from_cuda(launch_sort_quantize(q, ids, (int)pairs, d->experts, offsets, rows, st));
  } else {
    rc = from_cuda(launch_route_sort(ids, pairs, d->experts, offsets, rows, nullptr, (int32_t*)(ws + l.sort), st));
    if (rc == B2C_OK) rc = from_cuda(launch_fp8_quantize(q, st));
  }
  if (rc != B2C_OK) return rc;

  MatmulArgs m = {};
  m.a = q.q;
  m.lda = q.ldq;
  m.a_scale = q.scale;
  m.lds = q.lds;
  m.b = w1;
  m.b_scale = w1_scale;
  m.offsets = offsets;
  m.y = ws + l.hq;
  m.ldy = d->inter;
  m.y_scale = (float*)(ws + l.hs);
  m.ldys = blocks_of(d->inter);
  m.rows = (int)pairs;
  m.N = d->inter;
  m.K = d->hidden;
  m.groups = d->experts;
  m.a_type = m.b_type = m.y_type = B2C_E4M3;
  m.gated = 1;
  rc = launch_fp8_matmul(m, st);
  if (rc != B2C_OK) return rc;

  m.a = m.y;
  m.lda = m.ldy;
  m.a_scale = m.y_scale;
  m.lds = m.ldys;
  m.b = w2;
  m.b_scale = w2_scale;
  m.y = ws + l.y;
  m.ldy = d->hidden;
  m.y_scale = nullptr;
  m.ldys = 0;
  m.N = d->hidden;
  m.K = d->inter;
  // A slot's row is a partial sum: it stays in 32 bits, and y is rounded once.  (In the layer's type, half the traffic, 784 * 257 - 784 * 256
  // came out as 1024 in bf16 and NaN in f16; 8192 tokens, 4 of 64 experts, 2048 x 1024: 420 us instead of 379.)
  m.y_type = B2C_F32;
  m.gated = 0;
  m.early = 1;  // (the first product read its offsets after the sort had ended, and lets no later kernel start before that)
  rc = launch_fp8_matmul(m, st);
  if (rc != B2C_OK) return rc;
  return from_cuda(launch_route_combine(m.y, B2C_F32, pairs, m.ldy, rows, weights, tokens, d->topk, d->hidden, y, d->type, ldy, st));
}

int b2c_fp8_status(int32_t* status) {
  if (!status) return B2C_E_INVALID_ARG;
  return fp8_status_read_and_clear(status);
}

int b2c_selftest_fp8_wait(int form, void* cuda_stream) {
  if (form != 0 && form != 1) return B2C_E_INVALID_ARG;
  return from_cuda(form == 0 ? fp8_rows_wait_selftest((cudaStream_t)cuda_stream) : fp8_pair_wait_selftest((cudaStream_t)cuda_stream));
}

}  // extern "C"
