// C-ABI entry points of training in 8 bits (see include/t5mi.h): quantised matrices, their product, AdamW.
#include "block_host.h"
#include <memory>
#include <new>

namespace {

constexpr int kAdamMaxListed = 1 << 16;           // tensors one adamw_step_multi call may list
constexpr int64_t kAdamMost = (int64_t)1 << 34;   // elements of a tensor, and of a launch

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool fp8_type(int32_t t) { return t == T5_E4M3 || t == T5_E5M2; }
bool block_rows_ok(int32_t r) { return r == 1 || r == 128; }
int64_t blocks_of(int64_t n) { return (n + 127) / 128; }

int check_gemm(const t5_gemm_fp8_cfg* c) {
  if (!c) return T5_ERR_NULL;
  if (c->M < 0 || c->N < 1 || c->K < 1 || c->lda < c->K || c->ldb < c->K || c->ldc < c->N || c->lsa < blocks_of(c->K) ||
      c->lsb < blocks_of(c->K) || !block_rows_ok(c->a_block_rows) || !block_rows_ok(c->b_block_rows))
    return T5_ERR_SHAPE;
  if (!fp8_type(c->a_dtype) || !fp8_type(c->b_dtype) || (c->c_dtype != T5_F32 && c->c_dtype != T5_BF16) ||
      (c->accumulate && c->c_dtype != T5_F32))
    return T5_ERR_UNSUPPORTED;
  if (c->M > (1 << 30) || c->N > (1 << 30) || c->lda % 16 || c->ldb % 16 || c->lda > (1 << 23) || c->ldb > (1 << 23) ||
      c->lsa % 4 || c->lsb % 4 || c->lsa > (1 << 20) || c->lsb > (1 << 20) || c->ldc > ((int64_t)1 << 32))
    return T5_ERR_UNSUPPORTED;
  return T5_OK;
}

bool fraction(double b) { return b >= 0.0 && b < 1.0; }
bool positive(double x) { return x >= 0.0 && std::isfinite(x); }

int check_adam_tensor(const adamw_tensor& t) {
  if (t.n < 1 || !positive(t.weight_decay)) return T5_ERR_SHAPE;
  if (t.n > kAdamMost || (t.state_bits != 8 && t.state_bits != 32) || (t.grad_dtype != T5_F32 && t.grad_dtype != T5_BF16))
    return T5_ERR_UNSUPPORTED;
  if (!t.param || !t.grad || !t.m || !t.v || (t.state_bits == 8 && (!t.m_scale || !t.v_scale))) return T5_ERR_NULL;
  const uintptr_t state = t.state_bits == 8 ? 1 : 4;
  if (!aligned(t.param, 4) || !aligned(t.grad, t.grad_dtype == T5_BF16 ? 2 : 4) || !aligned(t.m, state) || !aligned(t.v, state) ||
      !aligned(t.bf16_copy_out, 2))
    return T5_ERR_UNSUPPORTED;
  return T5_OK;
}

// Whether two tensors of the list share parameters (an entry listed twice, say): two workgroups would update them at once.
int check_disjoint(const adamw_tensor* t, int n) {
  struct Range { uintptr_t from, to; };
  Range few[64];
  std::unique_ptr<Range[]> many(n > 64 ? new (std::nothrow) Range[n] : nullptr);
  Range* r = n > 64 ? many.get() : few;
  if (!r) return T5_ERR_DEVICE;  // no host memory
  for (int i = 0; i < n; ++i) r[i] = Range{(uintptr_t)t[i].param, (uintptr_t)t[i].param + (uintptr_t)t[i].n * 4};
  std::sort(r, r + n, [](const Range& a, const Range& b) { return a.from < b.from; });
  for (int i = 1; i < n; ++i)
    if (r[i].from < r[i - 1].to) return T5_ERR_SHAPE;
  return T5_OK;
}

}  // namespace

extern "C" {

int64_t t5_fp8_ld(int64_t cols) { return fp8_ld(cols); }
int64_t t5_fp8_scale_ld(int64_t cols) { return fp8_scale_ld(cols); }

int t5_quantize_fp8(const t5_quantize_cfg* cfg, const void* x, void* q, uint8_t* scale, void* qt, uint8_t* scale_t, void* stream) {
  if (!cfg) return T5_ERR_NULL;
  if (cfg->rows < 0 || cfg->cols < 1 || cfg->ld < cfg->cols || !block_rows_ok(cfg->block_rows)) return T5_ERR_SHAPE;
  if (cfg->rows > ((int64_t)1 << 31) - 129 || cfg->cols > (1 << 23) || cfg->ld > ((int64_t)1 << 32) ||
      (cfg->dtype != T5_F32 && cfg->dtype != T5_BF16) || !fp8_type(cfg->q_dtype))
    return T5_ERR_UNSUPPORTED;
  // (threads of a launch are numbered with 32 bits: 256 for 32 blocks of a row, 512 for a tile)
  if (qt || cfg->block_rows == 128 ? blocks_of(cfg->rows) * blocks_of(cfg->cols) >= (1 << 23) : cfg->rows * fp8_scale_ld(cfg->cols) >= (1 << 29))
    return T5_ERR_UNSUPPORTED;
  if (cfg->rows == 0) return T5_OK;
  if (!x || (!q && !qt) || !q != !scale || !qt != !scale_t) return T5_ERR_NULL;
  if (!aligned(x, cfg->dtype == T5_BF16 ? 2 : 4) || !aligned(q, 16) || !aligned(qt, 16) || !aligned(scale, 4) || !aligned(scale_t, 4))
    return T5_ERR_UNSUPPORTED;
  hipStream_t st = (hipStream_t)stream;
  T5_STEP("quantize_fp8", launch_quantize_fp8(*cfg, x, q, scale, qt, scale_t, st));
  return T5_OK;
}

size_t t5_gemm_fp8_workspace_bytes(const t5_gemm_fp8_cfg* cfg) {
  return check_gemm(cfg) == T5_OK && cfg->M > 0 ? gemm_fp8_ws_bytes(*cfg) : 0;
}

int t5_gemm_fp8_kernel_path(const t5_gemm_fp8_cfg* cfg) {
  return check_gemm(cfg) != T5_OK ? -1 : cfg->M > 0 ? gemm_fp8_path(*cfg) : 0;
}

int t5_gemm_fp8(const t5_gemm_fp8_cfg* cfg, const void* A, const uint8_t* a_scale, const void* B, const uint8_t* b_scale,
                void* C, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_gemm(cfg);
  if (rc != T5_OK) return rc;
  if (cfg->M == 0) return T5_OK;
  if (!A || !a_scale || !B || !b_scale || !C) return T5_ERR_NULL;
  if (!aligned(A, 16) || !aligned(B, 16) || !aligned(a_scale, 4) || !aligned(b_scale, 4) || !aligned(C, cfg->c_dtype == T5_BF16 ? 2 : 4))
    return T5_ERR_UNSUPPORTED;
  const size_t need = gemm_fp8_ws_bytes(*cfg);
  if (need > 0) {
    if (!workspace) return T5_ERR_NULL;
    if (workspace_bytes < need || !aligned(workspace, 256)) return T5_ERR_WORKSPACE;
  }
  hipStream_t st = (hipStream_t)stream;
  T5_STEP("gemm_fp8", launch_gemm_fp8(*cfg, A, a_scale, B, b_scale, C, workspace, st));
  return T5_OK;
}

int adamw_step_multi(const adamw_tensor* tensors, int n_tensors, const adamw_cfg* cfg, void* stream) {
  if (!tensors || !cfg) return T5_ERR_NULL;
  if (n_tensors < 1) return T5_ERR_SHAPE;
  if (n_tensors > kAdamMaxListed) return T5_ERR_UNSUPPORTED;
  if (cfg->step < 1 || !positive(cfg->lr) || !fraction(cfg->beta1) || !fraction(cfg->beta2) || !(cfg->eps >= 1e-30) ||
      !std::isfinite(cfg->eps))
    return T5_ERR_SHAPE;
  if (!aligned(cfg->grad_scale, 4)) return T5_ERR_UNSUPPORTED;
  for (int i = 0; i < n_tensors; ++i) {  // every entry is checked before the first launch
    const int rc = check_adam_tensor(tensors[i]);
    if (rc != T5_OK) return rc;
  }
  const int rc = check_disjoint(tensors, n_tensors);
  if (rc != T5_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  for (int i = 0; i < n_tensors;) {
    int m = 0;
    int64_t elements = 0;  // (threads of a launch are numbered with 32 bits, each has 8 elements)
    do elements += tensors[i + m++].n;
    while (m < kAdamTensors && i + m < n_tensors && elements + tensors[i + m].n <= kAdamMost);
    T5_STEP("adamw", launch_adamw(tensors + i, m, i, *cfg, st));
    i += m;
  }
  return T5_OK;
}

}  // extern "C"
