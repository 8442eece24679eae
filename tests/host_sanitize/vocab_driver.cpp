// Host-side check of the vocabulary operators of include/t5mi.h and the models that call them, as driver.cpp beside it
// (see tests/test_host_sanitizers_vocab.py).  Size queries and refusals over the whole range of every argument; and calls that
// pass the checks, for the arithmetic of their launches: the runtime's stand-ins turn every launch away, so these end with
// T5_ERR_DEVICE, and pointers are never followed.
#include <cmath>
#include <cstdio>
#include <cstring>
#include <limits>
#include <vector>
#include "../../include/t5mi.h"

static int failures = 0;
#define EXPECT(cond)                                                        \
  do {                                                                      \
    if (!(cond)) { std::printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #cond); ++failures; } \
  } while (0)

static void* const P = (void*)4096;  // 256-byte aligned, never followed
static float* const F = (float*)P;
static const int32_t* const I = (const int32_t*)P;
static const size_t kLots = (size_t)1 << 62;

static t5_block_cfg block(int B, int S, int d, int causal, int dtype) {
  t5_block_cfg c;
  std::memset(&c, 0, sizeof(c));
  c.batch = B; c.seq = S; c.d_model = d; c.n_heads = 2; c.d_kv = 16; c.d_ff = 64;
  c.num_buckets = 32; c.max_distance = 128; c.causal = causal; c.dtype = dtype;
  c.rms_eps = 1e-6f; c.attn_scale = 1.0f;
  return c;
}

static void embed() {
  const int64_t ns[] = {0, 1, 7, 777, 1024, 1025, 4096, 4097, 9001, 16384, 16385, 40000, 65537, 1000003, (1 << 24) - 1};
  const int32_t vs[] = {1, 2, 255, 257, 32128, 65536, 65537, 262144, 300000, 1 << 22}, ds[] = {1, 3, 4, 67, 768, 2048, 4100, 1 << 16};
  for (int64_t n : ns)
    for (int32_t v : vs)
      for (int32_t d : ds)
        for (int ty = 0; ty < 2; ++ty) {
          t5_embed_cfg c = {n, v, d, ty, 0.5f};
          const size_t need = t5_embed_bwd_workspace_bytes(&c);
          EXPECT(need >= 256);
          EXPECT(t5_embed_fwd(&c, I, P, P, nullptr) == (n ? T5_ERR_DEVICE : T5_OK));
          for (int acc = 0; acc < 2; ++acc) EXPECT(t5_embed_bwd(&c, I, P, F, acc, P, need, nullptr) == (n || !acc ? T5_ERR_DEVICE : T5_OK));
          EXPECT(t5_embed_bwd(&c, I, P, F, 0, P, need - 1, nullptr) == T5_ERR_WORKSPACE);
          EXPECT(t5_embed_bwd(&c, I, P, F, 0, (char*)P + 16, need, nullptr) == T5_ERR_WORKSPACE);
        }
  const t5_embed_cfg bad[] = {{-1, 8, 8, 0, 1.f}, {8, 0, 8, 0, 1.f}, {8, 8, 0, 0, 1.f}, {8, 8, 8, 0, NAN}, {8, 8, 8, 2, 1.f},
                              {INT64_MAX, 8, 8, 0, 1.f}, {8, INT32_MAX, 8, 0, 1.f}, {8, 8, INT32_MAX, 0, 1.f}, {INT64_MIN, INT32_MIN, INT32_MIN, -1, -1.f}};
  for (const auto& c : bad) {
    EXPECT(t5_embed_bwd_workspace_bytes(&c) == 0);
    EXPECT(t5_embed_fwd(&c, I, P, P, nullptr) > T5_ERR_NULL && t5_embed_bwd(&c, I, P, F, 0, P, kLots, nullptr) > T5_ERR_NULL);
  }
  EXPECT(t5_embed_fwd(nullptr, I, P, P, nullptr) == T5_ERR_NULL && t5_embed_bwd_workspace_bytes(nullptr) == 0);
}

static void rows() {
  const int64_t rs[] = {0, 1, 127, 128, 256, 257, 511, 512, 1024, 1025, 16384, (1 << 24) - 1};
  const int32_t vs[] = {2, 33, 256, 1000, 4100, 16385, 32769, 65537, 131072, 131073, 1000001, 1 << 22}, ks[] = {1, 32, 96, 97, 256};
  for (int64_t r : rs)
    for (int32_t v : vs)
      for (int32_t k : ks)
        for (int ty = 0; ty < 2; ++ty) {
          if (k > v) continue;
          const int64_t ld = r % 2 ? v : (int64_t)1 << 32;
          t5_top_logits_cfg t = {r, ld, v, k, ty};
          EXPECT(t5_top_logits(&t, P, F, (int32_t*)P, nullptr) == (r ? T5_ERR_DEVICE : T5_OK));
          t5_distill_cfg c = {r, ld, v, k, ty, 2.f, 0.5f, 1e-4f, r % 3 ? 0 : v + 1};
          const size_t need = t5_distill_workspace_bytes(&c);
          EXPECT(need >= 256);
          // (rows in parts: more workgroups than a launch can have are refused before it)
          EXPECT(t5_distill_loss_and_grad(&c, P, I, F, I, F, F, (char*)P + 4096, P, need, nullptr) == T5_ERR_DEVICE);
          EXPECT(t5_distill_loss_and_grad(&c, P, I, F, I, F, nullptr, nullptr, P, need, nullptr) == T5_ERR_DEVICE);
          EXPECT(t5_distill_loss_and_grad(&c, P, I, F, I, F, F, P, P, need - 1, nullptr) != T5_ERR_DEVICE);
          EXPECT(t5_distill_loss_and_grad(&c, P, I, F, I, F, F, nullptr, (char*)P + 64, need, nullptr) == T5_ERR_WORKSPACE);
        }
  const t5_distill_cfg ok = {8, 16, 16, 4, 1, 1.f, 0.5f, 0.f, 0};
  std::vector<t5_distill_cfg> bad(17, ok);
  bad[0].rows = -1; bad[1].ld = 15; bad[2].vocab = 1; bad[3].top_k = 0; bad[4].top_k = 17; bad[5].dtype = 9; bad[6].rows = INT64_MAX;
  bad[7].ld = INT64_MAX; bad[8].temperature = 0.f; bad[9].temperature = NAN; bad[10].temperature = 4e-39f; bad[11].soft_weight = 1.5f;
  bad[12].z_loss = -1.f; bad[13].z_loss = INFINITY; bad[14].dlogits_ld = 15; bad[15].dlogits_ld = INT64_MAX; bad[16].dlogits_ld = INT64_MIN;
  for (const auto& c : bad) {
    EXPECT(t5_distill_workspace_bytes(&c) == 0);
    EXPECT(t5_distill_loss_and_grad(&c, P, I, F, I, F, F, nullptr, P, kLots, nullptr) > T5_ERR_NULL);
  }
  EXPECT(t5_distill_workspace_bytes(nullptr) == 0 && t5_top_logits(nullptr, P, F, (int32_t*)P, nullptr) == T5_ERR_NULL);
}

static void models() {
  std::vector<t5_block_weights> lw(3);
  std::vector<t5_block_grads> lg(3);
  std::vector<t5_cross_weights> xw(3);
  std::vector<t5_cross_grads> xg(3);
  for (auto& w : lw) {
    std::memset(&w, 0, sizeof(w));
    w.ln1_scale = w.wq = w.wk = w.wv = w.wo = w.ln2_scale = w.wi0 = w.wi1 = w.wo_ff = P;
  }
  for (auto& g : lg) g.ln1_scale = g.wq = g.wk = g.wv = g.wo = g.rel_table = g.ln2_scale = g.wi0 = g.wi1 = g.wo_ff = F;
  for (auto& x : xw) x.lnx_scale = x.xq = x.xk = x.xv = x.xo = P;
  for (auto& x : xg) x.lnx_scale = x.xq = x.xk = x.xv = x.xo = F;
  const int vocabs[] = {2, 301, 512, 17000, 40000, 200000}, seqs[] = {1, 24, 128};
  for (int dtype = 0; dtype < 2; ++dtype)
    for (int tied = 0; tied < 2; ++tied)
      for (int V : vocabs)
        for (int S : seqs) {
          t5_stack_cfg c;
          std::memset(&c, 0, sizeof(c));
          c.block = block(130, S, 64, 1, dtype);
          c.n_layers = 3; c.vocab = V; c.tied_logits = tied; c.z_loss = 1e-4f;
          t5_distill_opts o = {V < 64 ? V : 64, 2.f, 0.5f};
          t5_stack_weights w = {P, P, lw.data(), P, tied ? nullptr : P};
          t5_stack_grads g = {F, F, lg.data(), F, tied ? nullptr : F};
          const size_t top = t5_stack_top_logits_workspace_bytes(&c, o.top_k), need = t5_stack_distill_workspace_bytes(&c, &o);
          EXPECT(top > 0 && need > t5_stack_workspace_bytes(&c));
          EXPECT(t5_stack_top_logits(&c, I, &w, o.top_k, F, (int32_t*)P, P, top, nullptr) == T5_ERR_DEVICE);
          EXPECT(t5_stack_top_logits(&c, I, &w, o.top_k, F, (int32_t*)P, P, top - 1, nullptr) == T5_ERR_WORKSPACE);
          EXPECT(t5_stack_distill_loss_and_grad(&c, &o, I, I, F, I, &w, F, &g, 0, P, need, nullptr) == T5_ERR_DEVICE);
          EXPECT(t5_stack_distill_loss_and_grad(&c, &o, I, I, F, I, &w, F, &g, 0, P, need - 1, nullptr) == T5_ERR_WORKSPACE);
          EXPECT(t5_stack_distill_loss_and_grad(&c, &o, I, I, F, I, &w, F, &g, 0, (char*)P + 128, need, nullptr) == T5_ERR_WORKSPACE);
          t5_encdec_cfg e;
          std::memset(&e, 0, sizeof(e));
          e.enc_block = block(130, 2 * S, 64, 0, dtype); e.dec_block = block(130, S, 64, 1, dtype);
          e.n_enc_layers = e.n_dec_layers = 3; e.vocab = V; e.tied_logits = tied;
          t5_encdec_weights ew = {P, P, lw.data(), P, P, lw.data(), xw.data(), P, tied ? nullptr : P};
          t5_encdec_grads eg = {F, F, lg.data(), F, F, lg.data(), xg.data(), F, tied ? nullptr : F};
          const size_t etop = t5_encdec_top_logits_workspace_bytes(&e, o.top_k), eneed = t5_encdec_distill_workspace_bytes(&e, &o);
          EXPECT(etop > 0 && eneed > t5_encdec_workspace_bytes(&e));
          EXPECT(t5_encdec_top_logits(&e, I, I, &ew, o.top_k, F, (int32_t*)P, P, etop, nullptr) == T5_ERR_DEVICE);
          EXPECT(t5_encdec_top_logits(&e, I, I, &ew, o.top_k, F, (int32_t*)P, (char*)P + 128, etop, nullptr) == T5_ERR_WORKSPACE);
          EXPECT(t5_encdec_distill_loss_and_grad(&e, &o, I, I, I, F, I, &ew, F, &eg, 1, P, eneed, nullptr) == T5_ERR_DEVICE);
          EXPECT(t5_encdec_distill_loss_and_grad(&e, &o, I, I, I, F, I, &ew, F, &eg, 1, P, eneed - 1, nullptr) == T5_ERR_WORKSPACE);
          o.top_k = V + 1;
          EXPECT(t5_stack_distill_workspace_bytes(&c, &o) == 0 && t5_encdec_distill_workspace_bytes(&e, &o) == 0);
          EXPECT(t5_stack_top_logits_workspace_bytes(&c, V + 1) == 0 && t5_encdec_top_logits_workspace_bytes(&e, -1) == 0);
        }
}

int main() {
  embed();
  rows();
  models();
  std::printf("%s: %d failure(s)\n", failures ? "FAILED" : "OK", failures);
  return failures ? 1 : 0;
}
