// Argument checks shared by the C-ABI entry points that take top logits or a teacher (vocab_ops.hip, stack.hip).
#pragma once
#include "block_host.h"

namespace {

bool aligned256(const void* workspace) { return ((uintptr_t)workspace & 255) == 0; }

int elem_type(int32_t dtype, int* ty) {
  if (dtype != T5_F32 && dtype != T5_BF16) return T5_ERR_UNSUPPORTED;
  *ty = dtype == T5_BF16 ? IN_BF16 : IN_F32;
  return T5_OK;
}

int check_rows(int64_t rows, int32_t vocab, int64_t ld, int32_t top_k) {
  if (rows < 0 || vocab < 2 || ld < vocab || top_k < 1 || top_k > vocab) return T5_ERR_SHAPE;
  if (rows >= (1 << 24) || vocab > (1 << 22) || ld > ((int64_t)1 << 32) || top_k > kTopMost) return T5_ERR_UNSUPPORTED;
  return T5_OK;
}

int check_top(const t5_top_logits_cfg* c, int* ty) {
  if (!c) return T5_ERR_NULL;
  const int rc = check_rows(c->rows, c->vocab, c->ld, c->top_k);
  return rc != T5_OK ? rc : elem_type(c->dtype, ty);
}

int check_distill(const t5_distill_cfg* c, int* ty) {
  if (!c) return T5_ERR_NULL;
  const int rc = check_rows(c->rows, c->vocab, c->ld, c->top_k);
  if (rc != T5_OK) return rc;
  // (1.44 = log2(e): the kernels' exponentials are powers of two of (x - max) * log2(e) / T: 0 times an infinite factor would be NaN)
  if (!(c->temperature > 0.f) || !std::isfinite(c->temperature) || !std::isfinite(1.4426950408889634f * (1.f / c->temperature)) ||
      !(c->soft_weight >= 0.f && c->soft_weight <= 1.f) || !(c->z_loss >= 0.f) || !std::isfinite(c->z_loss))
    return T5_ERR_SHAPE;
  if (c->dlogits_ld != 0 && c->dlogits_ld < c->vocab) return T5_ERR_SHAPE;
  if (c->dlogits_ld > ((int64_t)1 << 32)) return T5_ERR_UNSUPPORTED;
  return elem_type(c->dtype, ty);
}

}  // namespace
