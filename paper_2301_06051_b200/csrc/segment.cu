// dsvt_segment_attention and its backward pass: the calls' checks.
#include <math.h>

#include "segment.cuh"

namespace {
using namespace dsvt_train;

bool bad_rows(const void* p, int64_t ld, int64_t width, int size) {
  return !p || ((uintptr_t)p & 15) != 0 || ld < width || (ld * size) % 16 != 0;
}

int check(const dsvt_ctx* ctx, const dsvt_segment_attention_params* p, SegArgs* a) {
  if (!ctx || !p || p->n < 0 || p->heads < 1 || p->head_dim < 1 || !type_known(p->type)) return DSVT_ERR_INVALID_ARG;
  if (p->cap_segments < 0 || p->max_len < (p->n > 0 ? 1 : 0) || !(p->cap >= 0.f) || isinf(p->cap)) return DSVT_ERR_INVALID_ARG;
  // (a cap by which scale cannot be divided, or that is infinite in units of log 2, would make NaN of a score of zero)
  if (p->cap > 0.f && (isinf(p->scale / p->cap) || isinf(p->cap * kLog2e))) return DSVT_ERR_INVALID_ARG;
  if (p->head_dim % 8 != 0 || p->head_dim > kMaxDim || p->heads > kMaxHeads) return DSVT_ERR_UNSUPPORTED;
  if (p->n > ctx->max_voxels) return DSVT_ERR_CAPACITY;
  const int64_t width = (int64_t)p->heads * p->head_dim;
  const int size = type_size(p->type);
  if (p->n > 0) {
    if (bad_rows(p->q, p->ld_q, width, size) || bad_rows(p->k, p->ld_k, width, size) || bad_rows(p->v, p->ld_v, width, size))
      return DSVT_ERR_INVALID_ARG;
    if (!p->seg_start) return DSVT_ERR_INVALID_ARG;
  }
  const void* words[] = {p->order, p->seg_start, p->num_segments, p->bias};
  for (const void* q : words)
    if (((uintptr_t)q & 3) != 0) return DSVT_ERR_INVALID_ARG;
  a->q = p->q; a->k = p->k; a->v = p->v;
  a->ld_q = p->ld_q; a->ld_k = p->ld_k; a->ld_v = p->ld_v;
  a->order = p->order; a->seg_start = p->seg_start; a->num_segments = p->num_segments;
  a->n = p->n; a->heads = p->heads; a->dim = p->head_dim; a->cap_segments = p->cap_segments;
  a->max_len = p->max_len < p->n ? p->max_len : p->n;
  a->scale = p->scale; a->cap = p->cap;
  a->status = ctx->status;
  if (!p->bias) return DSVT_OK;
  if ((p->n > 0 && !p->coords) || ((uintptr_t)p->coords & 15) != 0 || !p->bucket_of || p->buckets < 1) return DSVT_ERR_INVALID_ARG;
  if (p->buckets > kMaxBuckets) return DSVT_ERR_UNSUPPORTED;
  int64_t low = 0, high = 0;
  int at = 0;
  for (int axis = 0; axis < 3; ++axis) {
    const int e = p->extent[axis];
    if (e < 1) return DSVT_ERR_INVALID_ARG;
    if (e > kMaxExtent) return DSVT_ERR_UNSUPPORTED;
    a->maps.extent[axis] = e;
    if (axis == 1) a->maps.at_y = at;
    if (axis == 2) a->maps.at_z = at;
    int lo = p->bucket_of[at], hi = lo;
    for (int i = 0; i < 2 * e - 1; ++i, ++at) {
      const int b = p->bucket_of[at];
      if (b < 0 || b >= p->buckets) return DSVT_ERR_INVALID_ARG;
      a->maps.of[at] = (uint16_t)b;
      if (b < lo) lo = b;
      if (b > hi) hi = b;
    }
    low += lo;
    high += hi;
  }
  if (low < 0 || high >= p->buckets) return DSVT_ERR_INVALID_ARG;
  a->bias = p->bias;
  a->coords = reinterpret_cast<const int4*>(p->coords);
  a->buckets = p->buckets;
  return DSVT_OK;
}

}  // namespace

extern "C" int dsvt_segment_attention(dsvt_ctx* ctx, const dsvt_segment_attention_params* params, void* out, int64_t ld_out) {
  SegArgs a = {};
  const int rc = check(ctx, params, &a);
  if (rc != DSVT_OK) return rc;
  if (a.n == 0) return DSVT_OK;
  if (bad_rows(out, ld_out, (int64_t)a.heads * a.dim, type_size(params->type))) return DSVT_ERR_INVALID_ARG;
  if (out == a.q || out == a.k || out == a.v) return DSVT_ERR_INVALID_ARG;
  if (a.cap_segments == 0) return DSVT_OK;
  a.out = out; a.ld_out = ld_out;
  DeviceGuard on(ctx->device);
  switch (params->type) {
    case DSVT_TYPE_F32: return launch_forward<float>(ctx, a);
    case DSVT_TYPE_BF16: return launch_forward<__nv_bfloat16>(ctx, a);
    default: return launch_forward<__half>(ctx, a);
  }
}

extern "C" int dsvt_segment_attention_backward(dsvt_ctx* ctx, const dsvt_segment_attention_params* params, const void* d_out,
                                               int64_t ld_dout, void* dq, int64_t ld_dq, void* dk, int64_t ld_dk, void* dv,
                                               int64_t ld_dv, float* dbias) {
  SegArgs a = {};
  const int rc = check(ctx, params, &a);
  if (rc != DSVT_OK) return rc;
  if (((uintptr_t)dbias & 3) != 0 || (dbias && !a.bias)) return DSVT_ERR_INVALID_ARG;
  if (dbias && (int64_t)a.heads * a.buckets > kMaxBiasTable) return DSVT_ERR_UNSUPPORTED;
  DeviceGuard on(ctx->device);
  if (a.n > 0) {
    const int64_t width = (int64_t)a.heads * a.dim;
    const int size = type_size(params->type);
    if (bad_rows(d_out, ld_dout, width, size) || bad_rows(dq, ld_dq, width, size) || bad_rows(dk, ld_dk, width, size) ||
        bad_rows(dv, ld_dv, width, size))
      return DSVT_ERR_INVALID_ARG;
    const void* in[] = {a.q, a.k, a.v, d_out};
    for (const void* p : in)
      if (dq == p || dk == p || dv == p) return DSVT_ERR_INVALID_ARG;
    if (dq == dk || dq == dv || dk == dv) return DSVT_ERR_INVALID_ARG;
  }
  if (a.n == 0 || a.cap_segments == 0) {
    if (dbias) DSVT_CUDA_TRY(ctx, cudaMemsetAsync(dbias, 0, (size_t)a.heads * a.buckets * sizeof(float), ctx->stream));
    return DSVT_OK;
  }
  a.d_out = d_out; a.ld_do = ld_dout;
  a.dq = dq; a.dk = dk; a.dv = dv; a.ld_dq = ld_dq; a.ld_dk = ld_dk; a.ld_dv = ld_dv;
  a.dbias = dbias;
  switch (params->type) {
    case DSVT_TYPE_F32: return launch_backward<float>(ctx, a);
    case DSVT_TYPE_BF16: return launch_backward<__nv_bfloat16>(ctx, a);
    default: return launch_backward<__half>(ctx, a);
  }
}
