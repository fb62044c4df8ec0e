// C-ABI front end of what stands around the layers (include/model/taw_model.h): argument validation and the launches.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "taw_internal.h"
#include "taw_status.h"

using namespace taw;

static constexpr int32_t kMaxRows = 1 << 24;      // tokens, vocabulary

static bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const char *p = static_cast<const char*>(a), *q = static_cast<const char*>(b);
  return na && nb && p < q + nb && q < p + na;
}
// bytes from the first element of a [rows, cols] matrix with row stride ld to behind its last one
static size_t span(int64_t rows, int64_t cols, int64_t ld, size_t e) { return rows > 0 ? (size_t)((rows - 1) * ld + cols) * e : 0; }

struct Piece {
  const void* p;
  size_t n;
};
// whether one of the first `written` pieces shares memory with another piece (NULL shares none)
template <size_t N>
static bool any_overlap(const Piece (&x)[N], size_t written) {
  for (size_t i = 0; i < written; ++i)
    for (size_t k = i + 1; k < N; ++k)
      if (x[i].p && x[k].p && overlap(x[i].p, x[i].n, x[k].p, x[k].n)) return true;
  return false;
}

static bool bad_dtype(int32_t d) { return d != TAW_F32 && d != TAW_BF16; }

static int check_ids(const void* ids, int32_t id_type, const char* what) {
  if (id_type != TAW_I32 && id_type != TAW_I64) return fail(TAW_ERR_DTYPE, "type %d of %s is neither TAW_I32 nor TAW_I64", id_type, what);
  if (!ids) return fail(TAW_ERR_NULL, "%s is NULL", what);
  if (reinterpret_cast<uintptr_t>(ids) % (id_type == TAW_I64 ? 8 : 4)) return fail(TAW_ERR_ALIGN, "%s is not aligned to its type", what);
  return TAW_OK;
}

// ------------------------------------------------------------------------------ embedding
static int check_embed(const taw_embed_desc* d, EmbedArgs* a) {
  if (!d) return fail(TAW_ERR_NULL, "desc is NULL");
  if (bad_dtype(d->dtype)) return fail(TAW_ERR_DTYPE, "dtype %d is neither TAW_F32 nor TAW_BF16", d->dtype);
  if (d->T < 0 || d->H <= 0 || d->V <= 0) return fail(TAW_ERR_SHAPE, "bad embedding shape (T=%d H=%d V=%d)", d->T, d->H, d->V);
  if (d->T > kMaxRows || d->V > kMaxRows || d->H > kMaxRows) return fail(TAW_ERR_SHAPE, "T=%d, H=%d or V=%d exceeds 2^24", d->T, d->H, d->V);
  if ((d->ld_table && d->ld_table < d->H) || (d->ld_x && d->ld_x < d->H)) return fail(TAW_ERR_SHAPE, "row stride smaller than H=%d", d->H);
  if (d->ld_table > (int64_t)1 << 32 || d->ld_x > (int64_t)1 << 32) return fail(TAW_ERR_SHAPE, "row stride exceeds 2^32");
  if (!std::isfinite(d->scale)) return fail(TAW_ERR_SHAPE, "scale is not finite");
  if (d->flags & ~TAW_ACCUMULATE) return fail(TAW_ERR_SHAPE, "unknown flag bits 0x%x", d->flags);
  *a = EmbedArgs{d->dtype, 0, d->T, d->H, d->V, d->ld_table ? d->ld_table : d->H, d->ld_x ? d->ld_x : d->H, d->scale, (d->flags & TAW_ACCUMULATE) ? 1 : 0};
  return TAW_OK;
}

extern "C" int taw_embed_fwd(const taw_embed_desc* desc, const void* ids, int32_t id_type, const void* table, void* x, void* stream) {
  EmbedArgs a;
  int rc = check_embed(desc, &a);
  if (rc) return rc;
  if (a.T == 0) return TAW_OK;
  rc = check_ids(ids, id_type, "ids");
  if (rc) return rc;
  a.id_type = id_type;
  TAW_REQUIRE_PTR(table); TAW_REQUIRE_PTR(x); TAW_REQUIRE_ALIGNED(table); TAW_REQUIRE_ALIGNED(x);
  const size_t e = dt_size(a.dtype), nx = span(a.T, a.H, a.ld_x, e);
  if (overlap(x, nx, table, span(a.V, a.H, a.ld_table, e)) || overlap(x, nx, ids, (size_t)a.T * (id_type == TAW_I64 ? 8 : 4)))
    return fail(TAW_ERR_SHAPE, "x overlaps the table or the ids");
  TAW_LAUNCH(launch_embed_fwd(a, ids, table, x, (hipStream_t)stream), "embedding");
  return TAW_OK;
}

extern "C" size_t taw_embed_bwd_workspace_bytes(const taw_embed_desc* desc) {
  EmbedArgs a;
  return check_embed(desc, &a) ? 0 : embed_bwd_workspace_bytes(a);
}

extern "C" int taw_embed_bwd(const taw_embed_desc* desc, const void* ids, int32_t id_type, const void* dx, float* G, void* workspace,
                             size_t workspace_bytes, void* stream) {
  EmbedArgs a;
  int rc = check_embed(desc, &a);
  if (rc) return rc;
  if (a.T == 0 && a.accumulate) return TAW_OK;
  a.id_type = id_type;
  if (a.T) {
    rc = check_ids(ids, id_type, "ids");
    if (rc) return rc;
    TAW_REQUIRE_PTR(dx);
    TAW_REQUIRE_ALIGNED(dx);
  }
  TAW_REQUIRE_PTR(G); TAW_REQUIRE_ALIGNED(G);
  const size_t need = embed_bwd_workspace_bytes(a);
  if (workspace_bytes < need) return fail(TAW_ERR_WORKSPACE, "workspace_bytes=%zu < required %zu", workspace_bytes, need);
  if (need) { TAW_REQUIRE_PTR(workspace); TAW_REQUIRE_ALIGNED(workspace); }
  const size_t nG = span(a.V, a.H, a.ld_table, 4), nd = span(a.T, a.H, a.ld_x, dt_size(a.dtype)), ni = (size_t)a.T * (id_type == TAW_I64 ? 8 : 4);
  if (overlap(G, nG, dx, nd) || overlap(G, nG, ids, ni) || overlap(workspace, need, G, nG) || overlap(workspace, need, dx, nd) || overlap(workspace, need, ids, ni))
    return fail(TAW_ERR_SHAPE, "buffers of the embedding's backward overlap");
  TAW_LAUNCH(launch_embed_bwd(a, ids, dx, G, workspace, (hipStream_t)stream), "embedding backward");
  return TAW_OK;
}

// ------------------------------------------------------------------------------ loss
static int check_loss(const taw_loss_desc* d, LossArgs* a) {
  if (!d) return fail(TAW_ERR_NULL, "desc is NULL");
  if (bad_dtype(d->dtype)) return fail(TAW_ERR_DTYPE, "dtype %d is neither TAW_F32 nor TAW_BF16", d->dtype);
  if (d->grad_dtype != d->dtype && d->grad_dtype != TAW_BF16) return fail(TAW_ERR_DTYPE, "grad_dtype must equal dtype or be TAW_BF16");
  const int V_pad = d->V_pad ? d->V_pad : d->V;
  if (d->T < 0 || d->V <= 0 || V_pad < d->V) return fail(TAW_ERR_SHAPE, "bad loss shape (T=%d V=%d V_pad=%d)", d->T, d->V, d->V_pad);
  if (d->T > kMaxRows || V_pad > kMaxRows) return fail(TAW_ERR_SHAPE, "T=%d or V_pad=%d exceeds 2^24", d->T, V_pad);
  const int64_t ld = d->ld ? d->ld : d->V, ldg = d->ld_grad ? d->ld_grad : V_pad;
  if (ld < d->V || ldg < V_pad) return fail(TAW_ERR_SHAPE, "row stride smaller than the row (ld=%lld V=%d ld_grad=%lld V_pad=%d)", (long long)d->ld, d->V, (long long)d->ld_grad, V_pad);
  if (ld > (int64_t)1 << 32 || ldg > (int64_t)1 << 32) return fail(TAW_ERR_SHAPE, "row stride exceeds 2^32");
  if (!(d->label_smoothing >= 0.f && d->label_smoothing < 1.f)) return fail(TAW_ERR_SHAPE, "need 0 <= label_smoothing < 1");
  if (!(d->z_loss >= 0.f && std::isfinite(d->z_loss))) return fail(TAW_ERR_SHAPE, "z_loss must be >= 0 and finite");
  if (!std::isfinite(d->grad_scale)) return fail(TAW_ERR_SHAPE, "grad_scale is not finite");
  if (d->flags & ~TAW_LOSS_MEAN) return fail(TAW_ERR_SHAPE, "unknown flag bits 0x%x", d->flags);
  *a = LossArgs{d->dtype, d->grad_dtype, 0, d->T, d->V, V_pad, ld, ldg, d->label_smoothing, d->z_loss, d->grad_scale, (d->flags & TAW_LOSS_MEAN) ? 1 : 0};
  return TAW_OK;
}

static size_t logits_bytes(const LossArgs& a) { return span(a.T, a.V, a.ld, dt_size(a.dtype)); }
static size_t dlogits_bytes(const LossArgs& a) { return span(a.T, a.V_pad, a.ld_grad, dt_size(a.grad_dtype)); }
static size_t label_bytes(const LossArgs& a) { return (size_t)a.T * (a.label_type == TAW_I64 ? 8 : 4); }

static int check_dlogits(const LossArgs& a, const void* logits, const void* dlogits) {
  if (overlap(logits, logits_bytes(a), dlogits, dlogits_bytes(a)) && !(logits == dlogits && a.dtype == a.grad_dtype && a.ld == a.ld_grad))
    return fail(TAW_ERR_SHAPE, "dlogits overlaps the logits and is not the logits, with their type and row stride");
  return TAW_OK;
}

extern "C" size_t taw_loss_workspace_bytes(const taw_loss_desc* desc) {
  LossArgs a;
  return check_loss(desc, &a) ? 0 : loss_workspace_bytes(a);
}

static int loss_call(const taw_loss_desc* desc, const void* logits, const void* labels, int32_t label_type, float* loss, float* loss_rows, float* lse,
                     void* dlogits, bool grad, void* workspace, size_t workspace_bytes, void* stream) {
  LossArgs a;
  int rc = check_loss(desc, &a);
  if (rc) return rc;
  a.label_type = label_type;
  if (a.T) {
    rc = check_ids(labels, label_type, "labels");
    if (rc) return rc;
    TAW_REQUIRE_PTR(logits); TAW_REQUIRE_ALIGNED(logits);
    if (grad) {
      TAW_REQUIRE_PTR(dlogits); TAW_REQUIRE_ALIGNED(dlogits);
      rc = check_dlogits(a, logits, dlogits);
      if (rc) return rc;
    }
  }
  TAW_REQUIRE_PTR(loss); TAW_REQUIRE_PTR(workspace);
  TAW_REQUIRE_ALIGNED(loss); TAW_REQUIRE_ALIGNED(workspace); TAW_REQUIRE_ALIGNED(loss_rows); TAW_REQUIRE_ALIGNED(lse);
  const size_t need = loss_workspace_bytes(a), rows = (size_t)a.T * 4;
  if (workspace_bytes < need) return fail(TAW_ERR_WORKSPACE, "workspace_bytes=%zu < required %zu", workspace_bytes, need);
  const Piece all[] = {{loss, 8}, {loss_rows, rows}, {lse, rows}, {workspace, need}, {labels, label_bytes(a)}, {logits, logits_bytes(a)}, {dlogits, grad ? dlogits_bytes(a) : 0}};
  if (any_overlap(all, 5)) return fail(TAW_ERR_SHAPE, "buffers of the loss overlap");
  TAW_LAUNCH(launch_loss(a, logits, labels, loss, loss_rows, lse, grad ? dlogits : nullptr, workspace, (hipStream_t)stream), "loss");
  return TAW_OK;
}

extern "C" int taw_loss_fwd(const taw_loss_desc* desc, const void* logits, const void* labels, int32_t label_type, float* loss, float* loss_rows, float* lse,
                            void* workspace, size_t workspace_bytes, void* stream) {
  return loss_call(desc, logits, labels, label_type, loss, loss_rows, lse, nullptr, false, workspace, workspace_bytes, stream);
}

extern "C" int taw_loss_fwd_bwd(const taw_loss_desc* desc, const void* logits, const void* labels, int32_t label_type, float* loss, float* loss_rows,
                                float* lse, void* dlogits, void* workspace, size_t workspace_bytes, void* stream) {
  return loss_call(desc, logits, labels, label_type, loss, loss_rows, lse, dlogits, true, workspace, workspace_bytes, stream);
}

extern "C" int taw_loss_bwd(const taw_loss_desc* desc, const void* logits, const void* labels, int32_t label_type, const float* lse, const float* dloss_rows,
                            void* dlogits, void* stream) {
  LossArgs a;
  int rc = check_loss(desc, &a);
  if (rc) return rc;
  if (a.T == 0) return TAW_OK;
  rc = check_ids(labels, label_type, "labels");
  if (rc) return rc;
  a.label_type = label_type;
  TAW_REQUIRE_PTR(logits); TAW_REQUIRE_PTR(lse); TAW_REQUIRE_PTR(dloss_rows); TAW_REQUIRE_PTR(dlogits);
  TAW_REQUIRE_ALIGNED(logits); TAW_REQUIRE_ALIGNED(lse); TAW_REQUIRE_ALIGNED(dloss_rows); TAW_REQUIRE_ALIGNED(dlogits);
  rc = check_dlogits(a, logits, dlogits);
  if (rc) return rc;
  const Piece all[] = {{dlogits, dlogits_bytes(a)}, {labels, label_bytes(a)}, {lse, (size_t)a.T * 4}, {dloss_rows, (size_t)a.T * 4}};
  if (any_overlap(all, 1)) return fail(TAW_ERR_SHAPE, "dlogits overlaps the labels or what is known of the rows");
  TAW_LAUNCH(launch_loss_bwd(a, logits, labels, lse, dloss_rows, dlogits, (hipStream_t)stream), "loss backward");
  return TAW_OK;
}

// ------------------------------------------------------------------------------ gradient norm and clipping
static int check_list(const taw_tensor* t, int32_t count) {
  if (count < 0) return fail(TAW_ERR_SHAPE, "count=%d is negative", count);
  if (count && !t) return fail(TAW_ERR_NULL, "tensors is NULL");
  for (int32_t i = 0; i < count; ++i) {
    if (bad_dtype(t[i].dtype)) return fail(TAW_ERR_DTYPE, "dtype %d of tensor %d is neither TAW_F32 nor TAW_BF16", t[i].dtype, i);
    if (t[i].n > (size_t)1 << 48) return fail(TAW_ERR_SHAPE, "tensor %d has more than 2^48 elements", i);
    if (t[i].n && !t[i].data) return fail(TAW_ERR_NULL, "data of tensor %d is NULL", i);
    if (!aligned16(t[i].data)) return fail(TAW_ERR_ALIGN, "data of tensor %d is not 16-byte aligned", i);
  }
  return TAW_OK;
}

static int check_clip(float max_norm, float grad_scale) {
  if (!(max_norm > 0.f)) return fail(TAW_ERR_SHAPE, "max_norm must be > 0");
  if (!std::isfinite(grad_scale)) return fail(TAW_ERR_SHAPE, "grad_scale is not finite");
  return TAW_OK;
}

extern "C" size_t taw_grad_norm_workspace_bytes(const taw_tensor* tensors, int32_t count) {
  return check_list(tensors, count) ? 0 : grad_norm_workspace_bytes(tensors, count);
}

static int sumsq_call(const taw_tensor* tensors, int32_t count, int set, int finish, float max_norm, float grad_scale, taw_clip_state* state, void* workspace,
                      size_t workspace_bytes, void* stream) {
  int rc = check_list(tensors, count);
  if (rc) return rc;
  TAW_REQUIRE_PTR(state); TAW_REQUIRE_PTR(workspace); TAW_REQUIRE_ALIGNED(state); TAW_REQUIRE_ALIGNED(workspace);
  const size_t need = grad_norm_workspace_bytes(tensors, count);
  if (workspace_bytes < need) return fail(TAW_ERR_WORKSPACE, "workspace_bytes=%zu < required %zu", workspace_bytes, need);
  if (overlap(state, sizeof(*state), workspace, need)) return fail(TAW_ERR_SHAPE, "the state overlaps the workspace");
  for (int32_t i = 0; i < count; ++i) {
    const size_t n = tensors[i].n * dt_size(tensors[i].dtype);
    if (overlap(tensors[i].data, n, state, sizeof(*state)) || overlap(tensors[i].data, n, workspace, need))
      return fail(TAW_ERR_SHAPE, "tensor %d overlaps the state or the workspace", i);
  }
  TAW_LAUNCH(launch_grad_sumsq(tensors, count, set, finish, max_norm, grad_scale, state, workspace, (hipStream_t)stream), "gradient norm");
  return TAW_OK;
}

extern "C" int taw_grad_norm(const taw_tensor* tensors, int32_t count, float max_norm, float grad_scale, taw_clip_state* state, void* workspace,
                             size_t workspace_bytes, void* stream) {
  int rc = check_clip(max_norm, grad_scale);
  return rc ? rc : sumsq_call(tensors, count, 1, 1, max_norm, grad_scale, state, workspace, workspace_bytes, stream);
}

extern "C" int taw_grad_sumsq(const taw_tensor* tensors, int32_t count, int32_t accumulate, taw_clip_state* state, void* workspace, size_t workspace_bytes,
                              void* stream) {
  return sumsq_call(tensors, count, accumulate ? 0 : 1, 0, 1.f, 1.f, state, workspace, workspace_bytes, stream);
}

extern "C" int taw_clip_coef(taw_clip_state* state, float max_norm, float grad_scale, void* stream) {
  int rc = check_clip(max_norm, grad_scale);
  if (rc) return rc;
  TAW_REQUIRE_PTR(state); TAW_REQUIRE_ALIGNED(state);
  TAW_LAUNCH(launch_clip_coef(max_norm, grad_scale, state, (hipStream_t)stream), "clip coefficient");
  return TAW_OK;
}

// whether two tensors of the list, or one and the state, share memory: each would be scaled twice, in no order
static int check_disjoint(const taw_tensor* t, int32_t count, const taw_clip_state* state) {
  const auto end = [&](const taw_tensor& x) { return static_cast<const char*>(x.data) + x.n * dt_size(x.dtype); };
  bool rising = true;
  const taw_tensor* last = nullptr;
  for (int32_t i = 0; i < count; ++i) {
    if (!t[i].n) continue;
    if (overlap(t[i].data, t[i].n * dt_size(t[i].dtype), state, sizeof(*state))) return fail(TAW_ERR_SHAPE, "tensor %d overlaps the state", i);
    rising = rising && (!last || static_cast<const char*>(t[i].data) >= end(*last));
    last = &t[i];
  }
  if (rising) return TAW_OK;
  try {
    std::vector<const taw_tensor*> by;
    for (int32_t i = 0; i < count; ++i)
      if (t[i].n) by.push_back(&t[i]);
    std::sort(by.begin(), by.end(), [](const taw_tensor* x, const taw_tensor* y) { return x->data < y->data; });
    for (size_t i = 1; i < by.size(); ++i)
      if (static_cast<const char*>(by[i]->data) < end(*by[i - 1]))
        return fail(TAW_ERR_SHAPE, "tensors %d and %d overlap", (int)(by[i - 1] - t), (int)(by[i] - t));
  } catch (const std::bad_alloc&) {
    return fail(TAW_ERR_UNSUPPORTED, "no host memory to look over %d tensors", count);
  }
  return TAW_OK;
}

extern "C" int taw_grad_clip(const taw_tensor* tensors, int32_t count, const taw_clip_state* state, void* stream) {
  int rc = check_list(tensors, count);
  if (rc) return rc;
  TAW_REQUIRE_PTR(state); TAW_REQUIRE_ALIGNED(state);
  rc = check_disjoint(tensors, count, state);
  if (rc) return rc;
  TAW_LAUNCH(launch_grad_clip(tensors, count, state, (hipStream_t)stream), "gradient clipping");
  return TAW_OK;
}

extern "C" int taw_optimizer_step_clipped(const taw_adamw_desc* opt, const taw_clip_state* state, void* W_chunk, int32_t chunk_dtype, float* master,
                                          float* m, float* v, float* G_shard, size_t n_elems, void* stream) {
  TAW_REQUIRE_PTR(state); TAW_REQUIRE_ALIGNED(state);
  const void* arrays[5] = {W_chunk, master, m, v, G_shard};
  for (int i = 0; i < 5; ++i)
    if (overlap(arrays[i], n_elems * (i == 0 && chunk_dtype == TAW_BF16 ? 2 : 4), state, sizeof(*state))) return fail(TAW_ERR_SHAPE, "an optimizer array overlaps the state");
  return optimizer_step(opt, state, W_chunk, chunk_dtype, master, m, v, G_shard, n_elems, (hipStream_t)stream);
}
