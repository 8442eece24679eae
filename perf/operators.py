"""Timed cases of the operators at the vocabulary ends of a stack, as a distillation run calls them.

Operators
  embed      t5_embed_fwd: scaled token embedding
  embed_bwd  t5_embed_bwd: gradient of the table, by sorted tokens
  top        t5_top_logits: the K largest logits of each row, as a teacher hands them on
  distill    t5_distill_loss_and_grad: loss against a teacher's top logits, hard targets and z-loss, with its gradient

Vocabulary 32128 and widths 64, 512, 768, 2048 are those of this repository's workloads; the other sizes are generic.
With own = False every operator is computed by elementary torch operations in 32 bits, rounded once at the end; with
own = True by the library's entry points.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "bf16": 2}
MOST_ELEMENTS = 1 << 26  # of a drawn case's gradient table or activations
MOST_LOGITS = 1 << 28    # of a drawn case's logits


def _embed(name, op, tokens, vocab, d, dtype, scale, pad=0.0):
    return dict(name=name, op=op, tokens=tokens, vocab=vocab, d=d, dtype=dtype, scale=scale, pad=pad)


def _top(name, rows, vocab, k, dtype, gap=0):
    return dict(name=name, op="top", rows=rows, vocab=vocab, k=k, dtype=dtype, gap=gap)


def _distill(name, rows, vocab, k, dtype, tau, soft, z, grad=True, gap=0):
    return dict(name=name, op="distill", rows=rows, vocab=vocab, k=k, dtype=dtype, tau=tau, soft=soft, z=z, grad=grad, gap=gap)


def listed():
    return [
        # one decoding step of eight sequences: nothing but latency
        _embed("embed_step", "embed", 8, 32128, 768, "bf16", math.sqrt(768.0)),
        # the input of a training step of the 12-layer language model, 32 x 512 tokens
        _embed("embed_base", "embed", 16384, 32128, 768, "bf16", math.sqrt(768.0)),
        # a toy model's step: no size is a round number, half of the batch is padding
        _embed("embed_bwd_small", "embed_bwd", 777, 509, 67, "f32", 1.0, 0.5),
        # the gradient of that language model's table, sequences padded by a seventh
        _embed("embed_bwd_base", "embed_bwd", 16384, 32128, 768, "bf16", math.sqrt(768.0), 0.14),
        # the widest layers of the repository, 32 x 1024 tokens, nothing padded
        _embed("embed_bwd_xl", "embed_bwd", 32768, 32128, 2048, "bf16", 1.0),
        # a teacher asked for the next token of eight sequences, logits in float32
        _top("top_step", 8, 32128, 16, "f32"),
        # a teacher's pass over a batch of 16 x 512 tokens
        _top("top_base", 8192, 32128, 64, "bf16"),
        # a vocabulary of an odd size in rows padded to a longer stride, float32
        _top("top_wide_odd", 1023, 100003, 100, "f32", 13),
        # a toy student's loss and gradient, odd vocabulary
        _distill("distill_small", 48, 509, 8, "f32", 1.0, 1.0, 0.0),
        # one chunk of logits of the language model: soft and hard targets mixed, temperature 2, z-loss
        _distill("distill_base", 16384, 32128, 64, "bf16", 2.0, 0.5, 1e-4),
        # few rows of a large vocabulary in float32: a fine-tuning step on short answers
        _distill("distill_wide", 200, 131071, 100, "f32", 1.5, 0.9, 1e-4, True, 1),
        # the validation loss alone
        _distill("distill_eval", 4096, 32128, 32, "bf16", 1.0, 0.7, 0.0, False),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("embed", "embed_bwd", "top", "distill"))
    dtype = rng.choice(("f32", "bf16", "bf16"))
    if op in ("embed", "embed_bwd"):
        d, vocab, tokens = _spread(rng, 32, 4096), _spread(rng, 200, 131072), _spread(rng, 1, 65536)
        if rng.random() < 0.6:
            d = -(-d // 64) * 64
        vocab = max(2, min(vocab, MOST_ELEMENTS // d))
        tokens = max(1, min(tokens, MOST_ELEMENTS // d))
        c = _embed("", op, tokens, vocab, d, dtype, rng.choice((1.0, math.sqrt(d), 0.37)), rng.choice((0.0, 0.1, 0.4)))
    else:
        vocab, rows = _spread(rng, 64, 131072), _spread(rng, 1, 16384)
        if rng.random() < 0.5:
            vocab = -(-vocab // 64) * 64
        rows = max(1, min(rows, MOST_LOGITS // vocab))
        k = min(_spread(rng, 1, 128), vocab // 2)
        gap = rng.choice((0, 0, 1, 24))
        if op == "top":
            c = _top("", rows, vocab, k, dtype, gap)
        else:
            c = _distill("", rows, vocab, k, dtype, rng.choice((1.0, 0.7, 2.0, 4.0)), rng.choice((1.0, 0.5, 0.9)),
                         rng.choice((0.0, 1e-4)), rng.random() < 0.75, gap)
    del c["name"]
    return c


def _tokens(g, n, vocab, pad):
    """Ids by a Zipf-like law, probability ~ 1 / (rank + 10), ranks dealt out at random; the last `pad` of every 512
    positions hold id 0."""
    u = torch.rand(n, device=DEV, generator=g, dtype=torch.float64)
    rank = (10.0 * ((1.0 + vocab / 10.0) ** u - 1.0)).long().clamp_(0, vocab - 1)
    ids = torch.randperm(vocab, device=DEV, generator=g)[rank].to(torch.int32)
    if pad > 0:
        ids[(torch.arange(n, device=DEV) % 512) >= round(512 * (1.0 - pad))] = 0
    return ids


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    if case["op"] in ("embed", "embed_bwd"):
        n, vocab, d = case["tokens"], case["vocab"], case["d"]
        s = dict(case=case, tokens=_tokens(g, n, vocab, case["pad"]))
        if case["op"] == "embed":
            s["table"] = torch.randn(vocab, d, device=DEV, generator=g, dtype=dt)
        else:
            s["dx"] = torch.randn(n, d, device=DEV, generator=g, dtype=dt) * 1e-2
        return s
    rows, vocab, k = case["rows"], case["vocab"], case["k"]
    wide = torch.randn(rows, vocab + case["gap"], device=DEV, generator=g, dtype=dt).mul_(2.5)
    s = dict(case=case, logits=wide[:, :vocab])
    if case["op"] == "distill":
        r = lambda hi: (torch.rand(rows, 1, device=DEV, generator=g) * hi).long()  # noqa: E731
        at = torch.arange(k, device=DEV)
        ids = (r(vocab) + at * (1 + r(vocab // k))) % vocab
        t = s["logits"].gather(1, ids).float() * 0.5 + 2.0 * torch.randn(rows, k, device=DEV, generator=g)
        held = torch.rand(rows, 1, device=DEV, generator=g)  # a few rows without a teacher, some with a short list
        ids = torch.where((held < 0.02) | ((held < 0.12) & (at >= (k + 1) // 2)), -1, ids)
        s["teacher_logits"], s["teacher_ids"] = t.sort(1, descending=True)[0], ids.to(torch.int32)
        tgt = (torch.rand(rows, device=DEV, generator=g) * vocab).to(torch.int32)
        s["targets"] = torch.where(torch.rand(rows, device=DEV, generator=g) < 0.1, -1, tgt)
    return s


def run(state):
    c = state["case"]
    if own:
        return _own(state, c)
    return {"embed": _plain_embed, "embed_bwd": _plain_embed_bwd, "top": _plain_top, "distill": _plain_distill}[c["op"]](state, c)


def _own(s, c):
    import paper_2203_17189_amd as P
    if c["op"] == "embed":
        return P.t5_embed_fwd(s["tokens"], s["table"], scale=c["scale"])
    if c["op"] == "embed_bwd":
        return P.t5_embed_bwd(s["tokens"], s["dx"], c["vocab"], scale=c["scale"])
    if c["op"] == "top":
        return P.t5_top_logits(s["logits"], c["k"])
    out = P.t5_distill_loss_and_grad(s["logits"], s["targets"], s["teacher_logits"], s["teacher_ids"], temperature=c["tau"],
                                     soft_weight=c["soft"], z_loss=c["z"], want_grads=c["grad"])
    return out if c["grad"] else out[:2]


def _plain_embed(s, c):
    return (s["table"][s["tokens"].long()].float() * c["scale"]).to(s["table"].dtype)


def _plain_embed_bwd(s, c):
    out = torch.zeros(c["vocab"], c["d"], device=DEV, dtype=torch.float32)
    return out.index_add_(0, s["tokens"].long(), s["dx"].float() * c["scale"])


def _plain_top(s, c):
    x = s["logits"].float() + 0.0
    b = x.view(torch.int32)
    b = b ^ ((b >> 31) & 0x7FFFFFFF)  # ordered as the values are
    key = (b.long() << 32) | (0xFFFFFFFF - torch.arange(c["vocab"], device=DEV))  # of equal ones the lowest id first
    ids = 0xFFFFFFFF - (key.topk(c["k"], dim=1, sorted=True)[0] & 0xFFFFFFFF)
    return x.gather(1, ids), ids.to(torch.int32)


def _log_softmax(x):
    x = x - x.amax(1, keepdim=True)
    return x - x.exp().sum(1, keepdim=True).log()


def _plain_distill(s, c):
    x, ids = s["logits"].float(), s["teacher_ids"].long()
    tau, soft, z = c["tau"], c["soft"], c["z"]
    counted = s["targets"] >= 0
    tgt = s["targets"].long().clamp(min=0)[:, None]
    n = counted.sum().clamp(min=1).float()
    held = ids >= 0
    any_held = held.any(1, keepdim=True)
    t = torch.where(held, s["teacher_logits"] / tau, -math.inf)
    t = torch.where(any_held, t, 0.0)
    log_p = _log_softmax(t)
    p = torch.where(held, log_p.exp(), 0.0)
    log_q1 = _log_softmax(x)
    log_q = log_q1 if tau == 1.0 else _log_softmax(x / tau)
    kl = torch.where(held & (p > 0), p * (log_p - log_q.gather(1, ids.clamp(min=0))), 0.0).sum(1)
    x_t, log_t = x.gather(1, tgt)[:, 0], log_q1.gather(1, tgt)[:, 0]
    lse = x_t - log_t
    row = (1.0 - soft) * -log_t + z * lse * lse + soft * tau * tau * kl
    row = torch.where(counted, row, 0.0)
    loss = (row.sum() / n).reshape(1)
    if not c["grad"]:
        return loss, row
    gain = torch.where(counted, 1.0 / n, 0.0)[:, None]
    dx = log_q1.exp() * ((1.0 - soft) + 2.0 * z * lse)[:, None]
    dx += log_q.exp() * (soft * tau * any_held)
    dx.scatter_add_(1, ids.clamp(min=0), -soft * tau * p)
    dx.scatter_add_(1, tgt, torch.full_like(tgt, -(1.0 - soft), dtype=torch.float32))
    return loss, row, (dx * gain).to(s["logits"].dtype)


def work(case):
    e = SIZES[case["dtype"]]
    if case["op"] == "embed":
        n = case["tokens"] * case["d"]
        return {"bytes": 2 * n * e + 4 * case["tokens"], "flops": n}
    if case["op"] == "embed_bwd":
        n = case["tokens"] * case["d"]
        return {"bytes": n * e + 4 * case["tokens"] + 4 * case["vocab"] * case["d"], "flops": 2 * n}
    n = case["rows"] * case["vocab"]
    if case["op"] == "top":
        return {"bytes": n * e + 8 * case["rows"] * case["k"], "flops": n}
    exps = 1 if case["tau"] == 1.0 else 2
    return {"bytes": n * e * (2 if case["grad"] else 1) + 8 * case["rows"] * (1 + case["k"]) + 4,
            "flops": n * exps * (4 if case["grad"] else 2)}


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "embed":
        return s["table"].to(f64)[s["tokens"].long()].mul_(case["scale"])
    if case["op"] == "embed_bwd":
        out = torch.zeros(case["vocab"], case["d"], device=DEV, dtype=f64)
        for i in range(0, case["tokens"], 8192):
            out.index_put_((s["tokens"][i:i + 8192].long(),), s["dx"][i:i + 8192].to(f64), accumulate=True)
        return out.mul_(case["scale"])
    x = s["logits"]
    if case["op"] == "top":
        return x.to(f64).sort(1, descending=True)[0][:, :case["k"]].contiguous(), None
    rows, dxs = [], []
    n = max(1, int((s["targets"] >= 0).sum()))
    tau, soft, z = case["tau"], case["soft"], case["z"]
    for i in range(0, case["rows"], 1024):
        xs, ids, tgt = x[i:i + 1024].to(f64), s["teacher_ids"][i:i + 1024].long(), s["targets"][i:i + 1024].long()
        lse1, lse_t = torch.logsumexp(xs, 1), torch.logsumexp(xs / tau, 1)
        t = s["teacher_logits"][i:i + 1024].to(f64) / tau
        w = torch.where(ids >= 0, torch.exp(t - t.amax(1, keepdim=True)), 0.0)
        total = w.sum(1, keepdim=True)
        p = torch.where(total > 0, w / total, 0.0)
        log_q = xs.gather(1, ids.clamp(min=0)) / tau - lse_t[:, None]
        kl = (torch.special.xlogy(p, p) - p * log_q).sum(1)
        at = torch.arange(len(tgt), device=DEV)
        on = (tgt >= 0).to(f64)
        hard = lse1 - xs[at, tgt.clamp(min=0)]
        rows.append(on * ((1 - soft) * hard + z * lse1 ** 2 + soft * tau ** 2 * kl))
        if case["grad"]:
            d = torch.exp(xs - lse1[:, None]) * (1 - soft + 2 * z * lse1)[:, None]
            d[at, tgt.clamp(min=0)] -= 1 - soft
            d += soft * tau * (total > 0) * torch.exp(xs / tau - lse_t[:, None])
            d.scatter_add_(1, ids.clamp(min=0), -soft * tau * p)
            dxs.append(d * (on / n)[:, None])
    row = torch.cat(rows)
    loss = (row.sum() / n).reshape(1)
    return (loss, row, torch.cat(dxs)) if case["grad"] else (loss, row)
