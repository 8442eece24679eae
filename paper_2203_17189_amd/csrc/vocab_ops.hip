// C-ABI entry points of the operators at the vocabulary ends of a stack (see include/t5mi.h): scaled embedding and
// its gradient, top logits, distillation loss.
#include "block_host.h"
#include "vocab_host.h"

namespace {

int check_embed(const t5_embed_cfg* c, int* ty) {
  if (!c) return T5_ERR_NULL;
  if (c->n_tokens < 0 || c->vocab < 1 || c->d_model < 1 || !std::isfinite(c->scale)) return T5_ERR_SHAPE;
  if (c->n_tokens >= (1 << 24) || c->vocab > (1 << 22) || c->d_model > (1 << 16)) return T5_ERR_UNSUPPORTED;
  return elem_type(c->dtype, ty);
}

struct DistillWs {
  float *n_counted, *row_loss;
  void* partial;
};
size_t carve_distill(const t5_distill_cfg* c, int ty, void* base, DistillWs* w) {
  Carver cv(base);
  w->n_counted = cv.take<float>(256);
  w->row_loss = cv.take<float>((size_t)c->rows * 4);
  w->partial = cv.take(distill_ws_bytes(c->rows, c->vocab, c->top_k, ty));
  return cv.off;
}

}  // namespace

extern "C" {

int t5_embed_fwd(const t5_embed_cfg* cfg, const int32_t* tokens, const void* table, void* x, void* stream) {
  int ty;
  const int rc = check_embed(cfg, &ty);
  if (rc != T5_OK) return rc;
  if (cfg->n_tokens == 0) return T5_OK;
  if (!tokens || !table || !x) return T5_ERR_NULL;
  hipStream_t st = (hipStream_t)stream;
  T5_STEP("embed_fwd", launch_embed_scaled_fwd(tokens, table, x, ty, cfg->n_tokens, cfg->d_model, cfg->vocab, cfg->scale, st));
  return T5_OK;
}

size_t t5_embed_bwd_workspace_bytes(const t5_embed_cfg* cfg) {
  int ty;
  if (check_embed(cfg, &ty) != T5_OK) return 0;
  return std::max<size_t>(256, embed_sorted_ws_bytes(cfg->n_tokens, cfg->vocab, cfg->d_model));
}

int t5_embed_bwd(const t5_embed_cfg* cfg, const int32_t* tokens, const void* dx, float* dtable, int accumulate,
                 void* workspace, size_t workspace_bytes, void* stream) {
  int ty;
  const int rc = check_embed(cfg, &ty);
  if (rc != T5_OK) return rc;
  if (cfg->n_tokens == 0 && accumulate) return T5_OK;
  if (!dtable || !workspace || (cfg->n_tokens > 0 && (!tokens || !dx))) return T5_ERR_NULL;
  if (workspace_bytes < t5_embed_bwd_workspace_bytes(cfg) || !aligned256(workspace)) return T5_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  T5_STEP("embed_bwd", launch_embed_sorted_bwd(tokens, dx, ty, dtable, cfg->n_tokens, cfg->d_model, cfg->vocab, cfg->scale,
                                               accumulate ? 1 : 0, workspace, st));
  return T5_OK;
}

int t5_top_logits(const t5_top_logits_cfg* cfg, const void* logits, float* values, int32_t* ids, void* stream) {
  int ty;
  const int rc = check_top(cfg, &ty);
  if (rc != T5_OK) return rc;
  if (cfg->rows == 0) return T5_OK;
  if (!logits || !values || !ids) return T5_ERR_NULL;
  hipStream_t st = (hipStream_t)stream;
  T5_STEP("top_logits", launch_top_logits(logits, ty, cfg->rows, cfg->vocab, cfg->ld, cfg->top_k, values, ids, st));
  return T5_OK;
}

size_t t5_distill_workspace_bytes(const t5_distill_cfg* cfg) {
  int ty;
  DistillWs w;
  if (check_distill(cfg, &ty) != T5_OK) return 0;
  return carve_distill(cfg, ty, nullptr, &w);
}

int t5_distill_loss_and_grad(const t5_distill_cfg* cfg, const void* logits, const int32_t* targets,
                             const float* teacher_logits, const int32_t* teacher_ids, float* loss, float* row_loss,
                             void* dlogits, void* workspace, size_t workspace_bytes, void* stream) {
  int ty;
  const int rc = check_distill(cfg, &ty);
  if (rc != T5_OK) return rc;
  if (!loss || !workspace) return T5_ERR_NULL;
  if (cfg->rows > 0 && (!logits || !teacher_logits || !teacher_ids || (!targets && cfg->soft_weight != 1.f)))
    return T5_ERR_NULL;
  const int64_t out_ld = cfg->dlogits_ld ? cfg->dlogits_ld : cfg->ld;
  if (dlogits && dlogits == logits && out_ld != cfg->ld) return T5_ERR_SHAPE;  // rows over others still to be read
  DistillWs w;
  if (workspace_bytes < carve_distill(cfg, ty, workspace, &w) || !aligned256(workspace)) return T5_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  DistillArgs a;
  a.targets = targets; a.teacher_logits = teacher_logits; a.teacher_ids = teacher_ids; a.n_counted = w.n_counted;
  a.all_targets = targets; a.all_rows = cfg->rows; a.partial = w.partial;
  a.row_loss = row_loss ? row_loss : w.row_loss;
  a.ld = cfg->ld; a.out_ld = out_ld; a.K = cfg->top_k; a.V = cfg->vocab;
  a.tau = cfg->temperature; a.inv_tau = 1.f / cfg->temperature; a.soft = cfg->soft_weight; a.z_loss = cfg->z_loss;
  if (dlogits) T5_STEP("distill_count", launch_distill_count(targets, cfg->rows, cfg->vocab, w.n_counted, st));
  T5_STEP("distill_rows", launch_distill_rows(a, logits, dlogits, ty, cfg->rows, st));
  T5_STEP("distill_mean", launch_distill_mean(a.row_loss, targets, cfg->rows, cfg->vocab, loss, st));
  return T5_OK;
}

}  // extern "C"
