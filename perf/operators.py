"""Performance cases of the operators at the two ends of a language model, whose gradients make
the largest buckets that a schedule has to place: the token embedding, the head with its softmax
cross entropy in pieces of the vocabulary, and distillation from a teacher's top logits.

A case is a dict of plain values.  `prepare` builds what a training or serving program holds
before the call, `run` is one pass: in plain torch operations in 32 bits, rounded once at the
end, or, where `own` is set, through the public binding.  `exact` is the definition in 64 bits.

Conventions of all cases: a token, label or teacher index of -1 stands for nothing (an empty slot
of a ragged batch, a position that is not trained on, an entry that the teacher did not keep);
what such a row gives is zero.  `row_grad` is the derivative of the program's loss by each row's
loss (one over the rows that count; for 16-bit floats times the loss scale).
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def _embed(name, n, vocab, hidden, dtype, grad, scale=1.0, pad=0, empty=0.0):
    return dict(name=name, op="embed", n=n, vocab=vocab, hidden=hidden, dtype=dtype, grad=grad, scale=scale, pad=pad,
                empty=empty)


def _head(name, n, vocab, hidden, dtype, grad, scale=1.0, pad=0, empty=0.0):
    return dict(name=name, op="head", n=n, vocab=vocab, hidden=hidden, dtype=dtype, grad=grad, scale=scale, pad=pad,
                empty=empty)


def _distill(name, n, vocab, top_k, dtype, grad, temperature=1.0, pad=0, empty=0.0):
    return dict(name=name, op="distill", n=n, vocab=vocab, top_k=top_k, dtype=dtype, grad=grad, temperature=temperature,
                pad=pad, empty=empty)


def listed():
    return [
        # one generated token on its way into the model: latency of a single lookup
        _embed("embed_one", 1, 50257, 1600, "bf16", False),
        # a training step's lookup, and the gradient of the whole table from the sorted tokens
        _embed("embed_train", 16384, 50257, 1600, "bf16", True),
        # the same with odd sizes in 32 bits, rows further apart than they are long, a scale, empty slots
        _embed("embed_odd", 4099, 32003, 1001, "f32", True, scale=31.64, pad=3, empty=0.1),
        # the log-probability of one generated token (serving)
        _head("head_score_one", 1, 50257, 1600, "bf16", False),
        # a few candidates scored together over a large vocabulary
        _head("head_score_few", 13, 131072, 4096, "bf16", False),
        # a small model trained in 32 bits
        _head("head_train_f32", 1024, 8209, 640, "f32", True),
        # odd sizes in 16-bit floats, a fifth of the positions not trained on
        _head("head_train_odd", 1003, 30011, 1021, "f16", True, scale=0.5, pad=5, empty=0.2),
        # the head of a training step on 8192 tokens
        _head("head_train", 8192, 50257, 1600, "bf16", True),
        # the same with a wide model and a large vocabulary
        _head("head_train_large", 8192, 131072, 4096, "bf16", True),
        # a handful of positions distilled, in 32 bits
        _distill("distill_few", 5, 50257, 32, "f32", True, temperature=2.0),
        # a training step's logits against the 64 logits kept of the teacher
        _distill("distill_train", 4096, 50257, 64, "bf16", True, temperature=2.0, empty=0.1),
        # a large odd vocabulary in 16-bit floats, rows of odd length one after the other
        _distill("distill_large", 8192, 131071, 128, "f16", True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("embed", "head", "head", "distill"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    pad = rng.choice((0, 0, 0, rng.randint(1, 9)))
    empty = rng.choice((0.0, 0.0, round(rng.uniform(0.02, 0.6), 2)))
    grad = rng.random() < 0.7
    vocab = _log(rng, 900, 131072)
    if op == "embed":
        n, hidden = _log(rng, 1, 16384), _log(rng, 64, 4096)
        hidden = min(hidden, 50257 * 1600 // vocab) if grad else hidden
        c = _embed("", n, vocab, hidden, dtype, grad, scale=rng.choice((1.0, round(math.sqrt(hidden), 3))), pad=pad, empty=empty)
    elif op == "head":
        n, hidden = _log(rng, 1, 8192), _log(rng, 64, 4096)
        if rng.random() < 0.5:   # most models' widths are whole multiples of 64
            hidden = max(64, hidden // 64 * 64)
        if dtype == "f32":       # models trained in 32 bits are the small ones
            n = min(n, 1 + int(2e10 / (vocab * hidden)))
        c = _head("", n, vocab, hidden, dtype, grad, scale=rng.choice((1.0, 1.0, 0.7)), pad=pad, empty=empty)
    else:
        n, top_k = _log(rng, 1, 8192), _log(rng, 1, 256)
        if dtype == "f32":
            n = min(n, 4096)
        c = _distill("", n, vocab, min(top_k, vocab), dtype, grad, temperature=rng.choice((1.0, 2.0, 4.0)), pad=pad, empty=empty)
    del c["name"]
    return c


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _rows(x, pad):
    """`x` with `pad` more elements between its rows, as a view of a wider buffer has them."""
    if not pad:
        return x
    wide = torch.zeros((x.shape[0], x.shape[1] + pad), dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


def _tokens(n, vocab, g):
    """Token numbers as text has them: the k-th most frequent one about 1/k as often as the first."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(vocab + 1.0)) - 1.0).long().clamp_(0, vocab - 1)


def _emptied(c, x, g):
    """`x` with the case's share of its rows set to -1 (never all of them)."""
    k = min(int(round(c["n"] * c["empty"])), c["n"] - 1)
    if k > 0:
        x[torch.randperm(c["n"], generator=g, device="cuda")[:k]] = -1
    return x


def _row_grad(c, valid):
    scale = 32768.0 if c["dtype"] == "f16" else 1.0
    return torch.where(valid, scale / valid.sum().clamp(min=1).float(), 0.0).float()


def prepare(case, seed):
    c, g, t = case, _gen(seed), TYPES[case["dtype"]]
    n, vocab = c["n"], c["vocab"]
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    s = {"case": c}
    if c["op"] == "embed":
        s["tokens"] = _emptied(c, _tokens(n, vocab, g), g).int()
        s["table"] = _rows((randn(vocab, c["hidden"]) * 0.02).to(t), c["pad"])
        if c["grad"]:
            s["grad_out"] = _rows((randn(n, c["hidden"]) * (16.0 if c["dtype"] == "f16" else 1e-3)).to(t), c["pad"])
    elif c["op"] == "head":
        labels = _tokens(n, vocab, g)
        w = randn(vocab, c["hidden"]) * (2.0 / math.sqrt(c["hidden"]))
        # a trained model's hidden states lean towards the row of the right token
        h = randn(n, c["hidden"]) + w[labels] * (2.0 * torch.rand((n, 1), generator=g, device="cuda"))
        s["labels"] = _emptied(c, labels, g).int()
        s["hidden"], s["weight"] = _rows(h.to(t), c["pad"]), _rows(w.to(t), c["pad"])
        if c["grad"]:
            s["row_grad"] = _row_grad(c, s["labels"] >= 0)
    else:
        x = torch.empty((n, vocab), dtype=t, device="cuda")
        step = max(1, (1 << 27) // vocab)
        index = torch.empty((n, c["top_k"]), dtype=torch.int32, device="cuda")
        value = torch.empty((n, c["top_k"]), device="cuda")
        for at in range(0, n, step):   # (in parts, so that 32-bit intermediates stay small)
            part = 2.5 * randn(min(step, n - at), vocab)
            x[at:at + step] = part.to(t)
            # the teacher: near the student on its better tokens, and sharper
            top = torch.topk(part + 0.7 * randn(part.shape[0], vocab), c["top_k"], dim=1)
            index[at:at + step], value[at:at + step] = top.indices.int(), 1.3 * top.values
        empty = _emptied(c, torch.zeros(n, dtype=torch.int64, device="cuda"), g) < 0
        index[empty] = -1
        if c["top_k"] > 1:   # some rows kept fewer than top_k
            index[torch.rand(n, generator=g, device="cuda") < 0.05, c["top_k"] // 2:] = -1
        s["logits"], s["teacher_index"], s["teacher_logit"] = _rows(x, c["pad"]), index, value
        if c["grad"]:
            s["row_grad"] = _row_grad(c, (index >= 0).any(dim=1))
    if own:
        from paper_2503_16815_amd import ends
        used = {"embed": ("embed", "embed_grad"), "head": ("head_loss", "head_grad"), "distill": ("distill",)}[c["op"]]
        s["ends"] = ends.DeftEnds(operators=used if c["grad"] else used[:1], dtype=t, max_rows=n, max_vocab=vocab,
                                  max_hidden=c.get("hidden", 0), max_top_k=c.get("top_k", 0))
    return s


def _plain_embed(c, s):
    tokens, scale, t = s["tokens"], c["scale"], s["table"].dtype
    valid = (tokens >= 0).unsqueeze(1)
    at = tokens.clamp(min=0).long()
    out = torch.where(valid, s["table"][at].float() * scale, 0.0).to(t)
    if not c["grad"]:
        return {"out": out}
    grad = torch.zeros(s["table"].shape, dtype=torch.float32, device=out.device)
    grad.index_add_(0, at, torch.where(valid, s["grad_out"].float() * scale, 0.0))
    return {"out": out, "grad_table": grad.to(t)}


def _plain_head(c, s):
    h, w, t = s["hidden"], s["weight"].float(), s["hidden"].dtype
    valid = s["labels"] >= 0
    at = s["labels"].clamp(min=0).long().unsqueeze(1)
    h = torch.where(valid.unsqueeze(1), h.float(), 0.0)
    z = (h @ w.T) * c["scale"]
    top = z.amax(dim=1, keepdim=True)
    lse = top + torch.exp(z - top).sum(dim=1, keepdim=True).log()
    loss = torch.where(valid, (lse - z.gather(1, at)).squeeze(1), 0.0)
    answer = {"loss": loss, "lse": torch.where(valid, lse.squeeze(1), 0.0)}
    if c["grad"]:
        rg = torch.where(valid, s["row_grad"], 0.0).unsqueeze(1)
        z = torch.exp(z - lse) * rg
        z.scatter_add_(1, at, -rg)
        answer["grad_hidden"] = ((z @ w) * c["scale"]).to(t)
        answer["grad_weight"] = ((z.T @ h) * c["scale"]).to(t)
    return answer


def _plain_distill(c, s):
    x, index, t = s["logits"], s["teacher_index"], s["logits"].dtype
    kept, at, inv = index >= 0, index.clamp(min=0).long(), 1.0 / c["temperature"]
    valid = kept.any(dim=1, keepdim=True)
    u = torch.where(kept, s["teacher_logit"] * inv, -math.inf)
    u = torch.where(valid, u - u.amax(dim=1, keepdim=True), 0.0)
    e = torch.where(kept, torch.exp(u), 0.0)
    total = e.sum(dim=1, keepdim=True)
    p = torch.where(valid, e / total, 0.0)
    log_p = u - total.log()
    z = x.float() * inv
    top = z.amax(dim=1, keepdim=True)
    lse = top + torch.exp(z - top).sum(dim=1, keepdim=True).log()
    by = torch.where(p > 0, p * (log_p - (z.gather(1, at) - lse)), 0.0)
    loss = torch.where(valid.squeeze(1), by.sum(dim=1) * c["temperature"] ** 2, 0.0)
    answer = {"loss": loss}
    if c["grad"]:
        rg = torch.where(valid, s["row_grad"].unsqueeze(1) * c["temperature"], 0.0)
        z = torch.exp(z - lse) * rg
        z.scatter_add_(1, at, -p * rg)
        answer["grad_logits"] = z.to(t)
    return answer


def _own_embed(c, s):
    ends = s["ends"]
    answer = {"out": ends.embed(s["tokens"], s["table"], scale=c["scale"])}
    if c["grad"]:
        answer["grad_table"] = ends.embed_grad(s["tokens"], s["grad_out"], vocab=c["vocab"], scale=c["scale"])
    return answer


def _own_head(c, s):
    ends = s["ends"]
    loss, lse = ends.head_loss(s["hidden"], s["weight"], s["labels"], logit_scale=c["scale"])
    answer = {"loss": loss, "lse": lse}
    if c["grad"]:
        answer["grad_hidden"], answer["grad_weight"] = ends.head_grad(
            s["hidden"], s["weight"], s["labels"], lse, s["row_grad"], logit_scale=c["scale"])
    return answer


def _own_distill(c, s):
    ends = s["ends"]
    if not c["grad"]:
        return {"loss": ends.distill(s["logits"], s["teacher_index"], s["teacher_logit"], temperature=c["temperature"])}
    loss, grad = ends.distill_grad(s["logits"], s["teacher_index"], s["teacher_logit"], s["row_grad"],
                                   temperature=c["temperature"])
    return {"loss": loss, "grad_logits": grad}


def run(state):
    form = {"embed": (_plain_embed, _own_embed), "head": (_plain_head, _own_head),
            "distill": (_plain_distill, _own_distill)}[state["case"]["op"]]
    return form[1 if own else 0](state["case"], state)


def work(case):
    """Each input read once, each output written once, and the products that the definition has: the
    logits, and for the gradients one product each for the hidden states and the weights."""
    c, b = case, BYTES[case["dtype"]]
    n, vocab = c["n"], c["vocab"]
    rows = n - min(int(round(n * c["empty"])), n - 1)
    if c["op"] == "embed":
        d = c["hidden"]
        bytes_ = 4 * n + b * d * (min(rows, vocab) + n)
        if c["grad"]:
            bytes_ += 4 * n + b * d * (rows + vocab)
        return {"bytes": bytes_, "flops": d * rows * (3 if c["grad"] else 1)}
    if c["op"] == "head":
        d = c["hidden"]
        bytes_ = b * d * (rows + vocab) + 12 * n
        flops = 2 * rows * vocab * d
        if c["grad"]:
            bytes_ += b * d * (n + vocab) + 4 * n
            flops *= 3
        return {"bytes": bytes_, "flops": flops}
    bytes_ = b * rows * vocab + 8 * n * c["top_k"] + 4 * n
    if c["grad"]:
        bytes_ += b * n * vocab + 4 * n
    return {"bytes": bytes_, "flops": rows * vocab * (6 if c["grad"] else 4)}


def _exact_embed(c, s):
    keep = (s["tokens"] >= 0).nonzero().squeeze(1)
    at = s["tokens"][keep].long()
    out = torch.zeros((c["n"], c["hidden"]), dtype=torch.float64, device="cuda")
    out[keep] = s["table"][at].double() * c["scale"]
    if not c["grad"]:
        return {"out": out}
    grad = torch.zeros((c["vocab"], c["hidden"]), dtype=torch.float64, device="cuda")
    grad.index_put_((at,), s["grad_out"][keep].double() * c["scale"], accumulate=True)
    return {"out": out, "grad_table": grad}


def _exact_head(c, s):
    keep = (s["labels"] >= 0).nonzero().squeeze(1)
    label = s["labels"][keep].long()
    w, f64 = s["weight"].double(), dict(dtype=torch.float64, device="cuda")
    loss, lse = torch.zeros(c["n"], **f64), torch.zeros(c["n"], **f64)
    grad_hidden, grad_weight = torch.zeros((c["n"], c["hidden"]), **f64), torch.zeros((c["vocab"], c["hidden"]), **f64)
    step = max(1, (1 << 28) // c["vocab"])
    for a in range(0, len(keep), step):
        rows, lab = keep[a:a + step], label[a:a + step]
        h = s["hidden"][rows].double()
        logp = torch.mm(h, w.t()).mul_(c["scale"])
        lse[rows] = torch.logsumexp(logp, dim=1)
        logp -= lse[rows][:, None]
        loss[rows] = -logp[torch.arange(len(rows), device="cuda"), lab]
        if c["grad"]:
            q = logp.exp_()
            q[torch.arange(len(rows), device="cuda"), lab] -= 1.0
            q *= (s["row_grad"][rows].double() * c["scale"])[:, None]
            grad_hidden[rows] = torch.mm(q, w)
            grad_weight += torch.mm(q.t(), h)
    answer = {"loss": loss, "lse": lse}
    return answer | ({"grad_hidden": grad_hidden, "grad_weight": grad_weight} if c["grad"] else {})


def _exact_distill(c, s):
    t = c["temperature"]
    loss = torch.zeros(c["n"], dtype=torch.float64, device="cuda")
    grad = torch.zeros((c["n"], c["vocab"]), dtype=torch.float64, device="cuda") if c["grad"] else None
    step = max(1, (1 << 26) // c["vocab"])
    for a in range(0, c["n"], step):
        z, index = s["logits"][a:a + step].double() / t, s["teacher_index"][a:a + step].long()
        has = (index >= 0).any(dim=1)
        u = (s["teacher_logit"][a:a + step].double() / t).masked_fill(index < 0, -math.inf)[has]
        p = torch.softmax(u, dim=1)
        log_q = torch.log_softmax(z[has], dim=1)
        at = index[has].clamp(min=0)
        part = torch.where(p > 0, p * (p.log() - log_q.gather(1, at)), 0.0).sum(dim=1)
        loss[a:a + step][has] = part * t * t
        if grad is not None:
            d = log_q.exp().scatter_add(1, at, -p)
            grad[a:a + step][has] = d * (s["row_grad"][a:a + step][has].double() * t)[:, None]
    return {"loss": loss} | ({"grad_logits": grad} if c["grad"] else {})


def exact(case, seed):
    asked = own
    globals()["own"] = False   # the inputs alone: no handle
    try:
        s = prepare(case, seed)
    finally:
        globals()["own"] = asked
    return {"embed": _exact_embed, "head": _exact_head, "distill": _exact_distill}[case["op"]](case, s)
