"""The operators at a language model's ends against their definitions in 64 bits.

Tolerances are error bounds, derived from the formulas and worked out element by element from the
inputs: u is half a unit in the last place of the output's type, e = 2^-24.
  embedding     one product in 32 bits, one rounding: (u + e) |x|; a sum of c rows: c e sum|x| on top
  logits        zerr = (hidden + 4) e sum_k |h_k w_k| |scale|
  softmax       lse: the largest zerr, and EXP for the exponentials and the order of the sum
                (an exponential of an argument down to -88 is off by 88 e and 2 e for the function; sums are
                a few hundred terms deep: together below 1e-4)
  derivative d  in 16 bits rounded once more (u |d|), else e; its softmax part is off by (2 zerr + EXP)
  products      sum of |errors of d| |w|, and the sum's own (terms e) sum |d w|
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
EXP = 1e-4
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}     # (bf16 and f16: half a unit is 2^-9, 2^-12; doubled for ties and scaling)
TINY = {"f32": 1e-37, "f16": 2.0 ** -24, "bf16": 1e-37}           # results below a type's smallest normal number
ALL = ("f32", "f16", "bf16")


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2503_16815_amd import ends
    ends.load_library()
    return torch


def handle(torch, ops, dtype, rows, vocab, hidden=0, top_k=0):
    from paper_2503_16815_amd import ends
    return ends.DeftEnds(ops, getattr(torch, {"f32": "float32", "f16": "float16", "bf16": "bfloat16"}[dtype]), max(1, rows), vocab,
                         hidden, top_k)


def matrix(torch, g, rows, width, dtype, scale=1.0, pad=0, shift=0):
    """A matrix of the type on the GPU; `pad` elements lie between rows, the first one `shift` elements past an
    aligned address; what lies between is NaN."""
    t = getattr(torch, {"f32": "float32", "f16": "float16", "bf16": "bfloat16"}[dtype])
    room = torch.full((rows * (width + pad) + shift + 16,), math.nan, dtype=t, device="cuda")
    m = room[shift:shift + rows * (width + pad)].view(rows, width + pad)[:, :width]
    m.copy_((torch.randn((rows, width), generator=g, device="cuda") * scale).to(t))
    return m


def generator(torch, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def within(got, want, bound, what):
    """Every element of `got` (finite) within `bound` of `want`, both in 64 bits."""
    got = got.double()
    assert got.shape == want.shape, what
    assert bool(got.isfinite().all()), what + ": not finite"
    over = ((got - want).abs() - bound).max() if got.numel() else 0.0
    assert float(over) <= 0.0, f"{what}: {float(over)} over its bound; largest error {float((got - want).abs().max())}"


# ---- embedding ------------------------------------------------------------------------------

def some_tokens(torch, g, n, vocab, kind):
    if kind == "same":
        return torch.full((n,), vocab - 1, dtype=torch.int32, device="cuda")
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    t = ((torch.exp(u * math.log(vocab + 1.0)) - 1.0).long().clamp(0, vocab - 1)).int()
    if kind == "ragged" and n > 1:
        t[torch.rand(n, generator=g, device="cuda") < 0.3] = -1
        t[n // 2] = vocab           # outside
        t[0] = -7                   # outside
    if kind == "empty":
        t[:] = -1
    return t


def embed_definition(torch, tokens, x, vocab):
    """Per vocabulary row, in 64 bits: the sum of its rows of x, the sum of their magnitudes and their number."""
    keep = ((tokens >= 0) & (tokens < vocab)).nonzero().squeeze(1)
    at = tokens[keep].long()
    total = torch.zeros((vocab, x.shape[1]), dtype=torch.float64, device="cuda").index_put_((at,), x[keep].double(), accumulate=True)
    mag = torch.zeros_like(total).index_put_((at,), x[keep].double().abs(), accumulate=True)
    count = torch.zeros(vocab, dtype=torch.float64, device="cuda").index_put_((at,), torch.ones(len(at), dtype=torch.float64, device="cuda"), accumulate=True)
    return total, mag, count


EMBED = [  # rows, vocab, hidden, pad, shift, tokens
    (1, 1, 1, 0, 0, "text"), (1, 50257, 64, 0, 0, "text"), (2, 3, 7, 1, 1, "same"), (31, 100, 8, 0, 0, "text"),
    (32, 100, 65, 3, 1, "same"), (33, 100, 129, 0, 1, "ragged"), (97, 17, 24, 0, 0, "ragged"), (500, 255, 200, 1, 0, "ragged"),
    (1000, 256, 96, 0, 0, "same"), (4096, 65536, 16, 0, 0, "text"), (4097, 65535, 33, 2, 3, "ragged"),
    (9001, 70000, 40, 0, 0, "ragged"), (64, 1000, 2056, 0, 0, "text"), (70, 9, 4099, 5, 1, "ragged"), (100, 50, 12, 0, 0, "empty"),
    (40000, 131072, 8, 0, 0, "ragged"),
]


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("rows,vocab,hidden,pad,shift,kind", EMBED)
def test_embedding(torch, dtype, rows, vocab, hidden, pad, shift, kind):
    g = generator(torch, rows * 7 + vocab)
    tokens = some_tokens(torch, g, rows, vocab, kind)
    table = matrix(torch, g, vocab, hidden, dtype, 0.5, pad, shift)
    dy = matrix(torch, g, rows, hidden, dtype, 1.0, pad, shift)
    dy[(tokens < 0) | (tokens >= vocab)] = math.nan        # nothing of these rows may come in
    scale = 1.7
    with handle(torch, ("embed", "embed_grad"), dtype, rows, vocab, hidden) as h:
        status = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
        out = h.embed(tokens, table, scale, status=status)
        valid = (tokens >= 0) & (tokens < vocab)
        want = torch.where(valid[:, None], table.double()[tokens.long().clamp(0, vocab - 1)] * scale, 0.0)
        within(out, want, (U[dtype] + 2 * E) * want.abs() + TINY[dtype], "embed")
        assert torch.equal(status, torch.where(valid | (tokens == -1), 0, 1).int())
        grad = h.embed_grad(tokens, dy, vocab=vocab, scale=scale)
        total, mag, count = embed_definition(torch, tokens, dy, vocab)
        bound = scale * mag * ((count[:, None] + 2) * E) + U[dtype] * (total * scale).abs() + TINY[dtype]
        within(grad, total * scale, bound, "embed_grad")
        assert bool((grad[count == 0] == 0).all())
        again = h.embed_grad(tokens, dy, vocab=vocab, scale=scale)
        assert torch.equal(grad, again)                    # one order of summation
        # merged into what is there: rows without a token keep their bits
        room = matrix(torch, g, vocab, hidden, dtype, 1.0, pad, shift)
        before = room.clone()
        h.embed_grad(tokens, dy, scale=scale, grad_table=room, accumulate=True)
        want = before.double() + total * scale
        within(room, want, bound + (U[dtype] + E) * want.abs() + E * before.double().abs(), "embed_grad, merged")
        assert torch.equal(room[count == 0], before[count == 0])


def test_embedding_of_no_rows(torch):
    with handle(torch, ("embed", "embed_grad"), "bf16", 4, 30, 8) as h:
        none = torch.empty(0, dtype=torch.int32, device="cuda")
        rows = torch.empty((0, 8), dtype=torch.bfloat16, device="cuda")
        table = torch.ones((30, 8), dtype=torch.bfloat16, device="cuda")
        assert h.embed(none, table).shape == (0, 8)
        h.embed_grad(none, rows, grad_table=table, accumulate=True)
        assert bool((table == 1).all())
        h.embed_grad(none, rows, grad_table=table)
        assert bool((table == 0).all())


def test_embedding_offsets_beyond_32_bits(torch):
    vocab, hidden, stride = 1 << 21, 24, 1100              # 2.3e9 elements
    room = torch.zeros(vocab * stride, dtype=torch.bfloat16, device="cuda").view(vocab, stride)[:, :hidden]
    tokens = torch.tensor([vocab - 1, 0, vocab - 2, vocab - 1], dtype=torch.int32, device="cuda")
    rows = torch.arange(4 * hidden, device="cuda").view(4, hidden).bfloat16()
    with handle(torch, ("embed", "embed_grad"), "bf16", 4, vocab, hidden) as h:
        h.embed_grad(tokens, rows, grad_table=room, accumulate=True)
        out = h.embed(tokens, room)
    assert torch.equal(out[1], rows[1]) and torch.equal(out[2], rows[2])
    want = rows[0].float() + rows[3].float()
    assert torch.equal(out[0], want.bfloat16()) and torch.equal(out[3], want.bfloat16())


# ---- head -----------------------------------------------------------------------------------

def head_definition(torch, h, w, labels, scale, row_grad, dtype, old=None):
    """Loss, lse, gradients in 64 bits, and the bounds on their errors."""
    vocab = w.shape[0]
    valid = (labels >= 0) & (labels < vocab)
    h, w = torch.where(valid[:, None], h.double(), 0.0), w.double()
    z = h @ w.T * scale
    zerr = ((h.abs() @ w.abs().T).amax(dim=1) * abs(scale) * (h.shape[1] + 4) * E)
    lse = torch.logsumexp(z, dim=1)
    at = labels.long().clamp(0, vocab - 1)[:, None]
    q = torch.exp(z - lse[:, None])
    rg = torch.where(valid, row_grad.double(), 0.0)[:, None]
    d = q.clone().scatter_add_(1, at, -torch.ones_like(at, dtype=torch.float64)) * rg
    derr = q * rg.abs() * (2 * zerr[:, None] + EXP) + d.abs() * (U[dtype] if dtype != "f32" else 4 * E) + rg.abs() * 1e-12
    gh, gw = d @ w * scale, d.T @ h * scale
    s = abs(scale)
    gh_err = (derr @ w.abs() + (d.abs() @ w.abs()) * (vocab + 32) * E) * s + U[dtype] * gh.abs() + TINY[dtype]
    gw_err = (derr.T @ h.abs() + (d.abs().T @ h.abs()) * (len(h) + 32) * E) * s + U[dtype] * gw.abs() + TINY[dtype]
    if old is not None:
        gw = gw + old.double()
        gw_err = gw_err + (U[dtype] + E) * gw.abs() + E * old.double().abs()
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    loss = torch.where(valid, lse - z.gather(1, at).squeeze(1), zero)
    loss_err = torch.where(valid, 2 * zerr + EXP + 4 * E * lse.abs(), zero)
    return valid, (loss, loss_err), (torch.where(valid, lse, zero), loss_err), (gh, gh_err), (gw, gw_err)


HEAD = [  # rows, vocab, hidden, pad, shift, scale, empty
    (1, 1, 1, 0, 0, 1.0, 0.0), (1, 50257, 64, 0, 0, 1.0, 0.0), (2, 5, 3, 1, 1, 0.5, 0.0), (3, 300, 64, 0, 0, 1.0, 0.4),
    (15, 64, 128, 0, 0, 1.0, 0.0), (16, 257, 96, 2, 1, 2.0, 0.3), (17, 1000, 192, 64, 0, 1.0, 0.0), (63, 255, 65, 0, 0, 1.0, 0.2),
    (64, 256, 64, 0, 0, 1.0, 0.0), (65, 513, 320, 8, 0, -1.0, 0.3), (128, 700, 128, 0, 0, 1.0, 0.0), (129, 1300, 72, 0, 0, 1.0, 0.5),
    (256, 2048, 256, 0, 0, 1.0, 0.0), (257, 2049, 257, 1, 1, 1.0, 0.1), (600, 4100, 512, 0, 0, 1.0, 0.7), (1030, 30, 64, 0, 0, 1.0, 0.1),
    (700, 1027, 1000, 4, 2, 1.0, 0.2),
]


def head_inputs(torch, seed, rows, vocab, hidden, pad, shift, empty, dtype):
    g = generator(torch, seed)
    h = matrix(torch, g, rows, hidden, dtype, 1.0, pad, shift)
    w = matrix(torch, g, vocab, hidden, dtype, 2.0 / math.sqrt(hidden), pad, shift)
    labels = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    labels[torch.rand(rows, generator=g, device="cuda") < empty] = -1
    row_grad = torch.rand(rows, generator=g, device="cuda") * (64.0 if dtype == "f16" else 1.0)
    return h, w, labels, row_grad


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("rows,vocab,hidden,pad,shift,scale,empty", HEAD)
def test_head(torch, dtype, rows, vocab, hidden, pad, shift, scale, empty):
    h, w, labels, row_grad = head_inputs(torch, rows + vocab, rows, vocab, hidden, pad, shift, empty, dtype)
    if rows > 4 and empty:
        labels[rows // 3] = vocab + 4                      # outside
    old = matrix(torch, generator(torch, 5), vocab, hidden, dtype, 1.0, pad, shift)
    valid, loss, lse, gh, gw = head_definition(torch, h, w, labels, scale, row_grad, dtype)
    for t in (h, row_grad):                                # masked rows may hold anything
        t[~valid] = math.nan
    with handle(torch, ("head_loss", "head_grad"), dtype, rows, vocab, hidden) as e:
        status = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
        got_loss, got_lse = e.head_loss(h, w, labels, scale, status=status)
        within(got_loss, *loss, "loss")
        within(got_lse, *lse, "lse")
        assert torch.equal(status, torch.where(valid | (labels == -1), 0, 1).int())
        got_gh, got_gw = e.head_grad(h, w, labels, got_lse, row_grad, scale)
        within(got_gh, *gh, "grad_hidden")
        within(got_gw, *gw, "grad_weight")
        assert bool((got_gh[~valid] == 0).all())
        alone, none = e.head_grad(h, w, labels, got_lse, row_grad, scale, need_weight=False)
        assert none is None and torch.equal(alone, got_gh)
        none, alone = e.head_grad(h, w, labels, got_lse, row_grad, scale, need_hidden=False)
        assert none is None and torch.equal(alone, got_gw)
        merged = old.clone() if pad == 0 else old
        _, merged_want = head_definition(torch, torch.where(valid[:, None], h, 0), w, labels, scale,
                                         torch.where(valid, row_grad, 0), dtype, old)[3:]
        e.head_grad(h, w, labels, got_lse, row_grad, scale, grad_weight=merged, accumulate=True)
        within(merged, *merged_want, "grad_weight, merged")


@pytest.mark.parametrize("dtype", ALL)
def test_head_without_any_label(torch, dtype):
    h, w, labels, row_grad = head_inputs(torch, 3, 70, 300, 64, 0, 0, 0.0, dtype)
    labels[:] = -1
    h[:] = math.nan
    with handle(torch, ("head_loss", "head_grad"), dtype, 70, 300, 64) as e:
        loss, lse = e.head_loss(h, w, labels)
        gh, gw = e.head_grad(h, w, labels, lse, row_grad)
    assert all(bool((x == 0).all()) for x in (loss, lse, gh, gw))


def test_head_of_no_rows(torch):
    with handle(torch, ("head_loss", "head_grad"), "bf16", 4, 30, 8) as e:
        h = torch.empty((0, 8), dtype=torch.bfloat16, device="cuda")
        w = torch.ones((30, 8), dtype=torch.bfloat16, device="cuda")
        none = torch.empty(0, device="cuda")
        loss, lse = e.head_loss(h, w, none.int())
        gw = torch.ones((30, 8), dtype=torch.bfloat16, device="cuda")
        e.head_grad(h, w, none.int(), none, none, grad_weight=gw, accumulate=True)
        assert len(loss) == 0 and bool((gw == 1).all())
        e.head_grad(h, w, none.int(), none, none, grad_weight=gw)
        assert bool((gw == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_head_in_several_pieces(torch, dtype):
    """A vocabulary that takes several pieces (the handle's limit on rows makes them small)."""
    from paper_2503_16815_amd import ends
    rows, vocab, hidden = 300, 5000, 72
    h, w, labels, row_grad = head_inputs(torch, 8, rows, vocab, hidden, 0, 0, 0.2, dtype)
    valid, loss, lse, gh, gw = head_definition(torch, h, w, labels, 1.0, row_grad, dtype)
    with ends.DeftEnds(("head_loss", "head_grad"), h.dtype, 1 << 17, vocab, hidden) as e:
        piece = e.info().vocab_piece
        assert piece < vocab / 2
        events = [torch.cuda.Event() for _ in range(-(-vocab // piece))]
        got_loss, got_lse = e.head_loss(h, w, labels)
        got_gh, got_gw = e.head_grad(h, w, labels, got_lse, row_grad, piece_events=events)
        other = torch.cuda.Stream()
        copies = []
        with torch.cuda.stream(other):                     # a bucket leaves as soon as its piece is final
            for i, ev in enumerate(events):
                other.wait_event(ev)
                copies.append(got_gw[i * piece:(i + 1) * piece].clone())
        other.synchronize()
        assert torch.equal(torch.cat(copies), got_gw)
        torch.cuda.synchronize()
        within(got_loss, *loss, "loss")
        within(got_gh, *gh, "grad_hidden")
        within(got_gw, *gw, "grad_weight")


def test_head_gradient_against_differences(torch):
    rows, vocab, hidden, eps = 9, 130, 33, 2e-2
    h, w, labels, row_grad = head_inputs(torch, 11, rows, vocab, hidden, 0, 0, 0.2, "f32")
    g = generator(torch, 12)
    row_grad[labels < 0] = 0.0
    with handle(torch, ("head_loss", "head_grad"), "f32", rows, vocab, hidden) as e:
        total = lambda hh, ww: float((e.head_loss(hh, ww, labels)[0].double() * row_grad.double()).sum())  # noqa: E731
        gh, gw = e.head_grad(h, w, labels, e.head_loss(h, w, labels)[1], row_grad)
        for _ in range(4):
            dh, dw = torch.randn(h.shape, generator=g, device="cuda"), torch.randn(w.shape, generator=g, device="cuda") / 6
            for (by, slope) in (((dh, torch.zeros_like(w)), (gh * dh).double().sum()), ((torch.zeros_like(h), dw), (gw * dw).double().sum())):
                f = lambda t: total(h + t * by[0], w + t * by[1])  # noqa: E731
                # fourth-order difference: its own error is eps^4 / 30 times the fifth derivative (logits move by
                # a few per unit of t: below 1e-4), that of the losses 1e-6 / eps of their sum
                diff = (8 * (f(eps) - f(-eps)) - (f(2 * eps) - f(-2 * eps))) / (12 * eps)
                assert abs(diff - float(slope)) <= 2e-3 * (1 + abs(float(slope)))


def test_head_offsets_beyond_32_bits(torch):
    vocab, hidden, stride = 1 << 21, 64, 1104
    room = torch.zeros(vocab * stride, dtype=torch.bfloat16, device="cuda").view(vocab, stride)[:, :hidden]
    h = torch.ones((2, hidden), dtype=torch.bfloat16, device="cuda")
    room[vocab - 1] = 0.25                                  # one logit of 16, the others 0
    labels = torch.tensor([vocab - 1, 7], dtype=torch.int32, device="cuda")
    with handle(torch, ("head_loss", "head_grad"), "bf16", 2, vocab, hidden) as e:
        loss, lse = e.head_loss(h, room, labels)
        want = math.log(vocab - 1 + math.exp(16.0))
        assert abs(float(lse[0]) - want) < EXP and abs(float(loss[0]) - (want - 16)) < EXP and abs(float(loss[1]) - want) < EXP
        out = torch.empty((vocab, stride), dtype=torch.bfloat16, device="cuda")[:, :hidden]
        gh, _ = e.head_grad(h, room, labels, lse, torch.ones(2, device="cuda"), grad_weight=out)
        p = math.exp(16.0 - want)
        assert abs(float(gh[0, 3]) - 0.25 * (p - 1)) < 2e-3 and abs(float(gh[1, 3]) - 0.25 * p) < 2e-3
        assert abs(float(out[vocab - 1, 5]) - (2 * p - 1)) < 8e-3 and abs(float(out[7, 5]) + 1) < 8e-3
        # all of a position's derivative sums to zero: the other rows' parts are there too
        assert abs(float(out[:, 9].float().sum())) < 0.05


def test_head_of_extreme_logits(torch):
    """Logits that are huge, equal, or the type's lowest value."""
    low = torch.finfo(torch.bfloat16).min
    w = torch.zeros((300, 64), dtype=torch.bfloat16, device="cuda")
    w[:, 0] = torch.linspace(-100, 100, 300).bfloat16()
    w[17, 1] = low
    h = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    h[0, 0], h[1, 0], h[3, 1] = 100.0, -100.0, 1.0          # row 2: all logits 0; row 3: one is the lowest value
    labels = torch.tensor([299, 5, 3, 17], dtype=torch.int32, device="cuda")
    z = h.double() @ w.double().T
    with handle(torch, ("head_loss", "head_grad"), "bf16", 4, 300, 64) as e:
        loss, lse = e.head_loss(h, w, labels)
        want = torch.logsumexp(z, 1)
        assert bool(((lse.double() - want).abs() <= EXP + 1e-6 * want.abs()).all())
        per = want - z.gather(1, labels.long()[:, None]).squeeze(1)
        assert bool(((loss.double() - per).abs() <= 2 * EXP + 1e-6 * per.abs()).all())
        gh, gw = e.head_grad(h, w, labels, lse, torch.ones(4, device="cuda"))
        q = torch.softmax(z, 1)
        q[torch.arange(4), labels.long()] -= 1
        within(gw, q.T @ h.double(), 0.01 * (q.abs().T @ h.double().abs()) + EXP, "grad_weight")


# ---- distillation ---------------------------------------------------------------------------

def distill_definition(torch, z, index, value, t, row_grad, dtype):
    vocab = z.shape[1]
    kept = index >= 0
    valid = kept.any(dim=1)
    u = torch.where(kept, value.double() / t, -math.inf)
    u[~valid] = 0.0
    p = torch.softmax(u, dim=1) * kept
    zz = torch.where(valid[:, None], z.double() / t, 0.0)
    log_q = torch.log_softmax(zz, dim=1)
    at = index.long().clamp(min=0)
    log_p = torch.log_softmax(u, dim=1)
    terms = torch.where(p > 0, p * (log_p - log_q.gather(1, at)), 0.0)
    size = torch.where(p > 0, p * (log_p.abs() + log_q.gather(1, at).abs() + 1), 0.0).sum(1)
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    loss = torch.where(valid, terms.sum(1) * t * t, zero)
    loss_err = torch.where(valid, t * t * size * 3 * EXP, zero)
    g = torch.where(valid, row_grad.double(), zero)[:, None] * t
    q = log_q.exp()
    d = q.scatter_add(1, at, -p) * g
    spread = torch.zeros_like(q).scatter_add(1, at, p)
    err = g.abs() * EXP * (2 * q + spread) + U[dtype] * d.abs() + TINY[dtype]
    return valid, (loss, loss_err), (d, err)


DISTILL = [  # rows, vocab, top_k, pad, shift, temperature
    (1, 1, 1, 0, 0, 1.0), (2, 7, 3, 1, 1, 2.0), (3, 8, 8, 0, 0, 1.0), (5, 511, 17, 0, 1, 0.5), (4, 4096, 64, 0, 0, 2.0),
    (9, 4097, 63, 3, 0, 4.0), (7, 12345, 100, 0, 3, 1.0), (3, 50257, 32, 0, 0, 2.0), (2, 65537, 1024, 1, 0, 1.0),
    (2, 131071, 256, 0, 0, 2.0), (2, 200001, 513, 2, 1, 1.0), (300, 1000, 5, 0, 0, 1.0), (2, 600000, 9, 0, 0, 3.0),
]


@pytest.mark.parametrize("dtype", ALL)
@pytest.mark.parametrize("rows,vocab,top_k,pad,shift,t", DISTILL)
def test_distillation(torch, dtype, rows, vocab, top_k, pad, shift, t):
    g = generator(torch, rows * 3 + vocab)
    z = matrix(torch, g, rows, vocab, dtype, 2.5, pad, shift)
    order = torch.stack([torch.randperm(vocab, generator=g, device="cuda")[:top_k] for _ in range(rows)])
    index = order.int()
    value = torch.randn((rows, top_k), generator=g, device="cuda") * 3
    index[torch.rand((rows, top_k), generator=g, device="cuda") < 0.2] = -1
    if top_k > 2:
        index[0, 2] = index[0, 0]                          # an index that occurs twice
    if rows > 1:
        index[rows - 1] = -1                               # a row of which nothing was kept
        z[rows - 1] = math.nan
    value[index < 0] = math.nan
    row_grad = torch.rand(rows, generator=g, device="cuda") * 2
    if rows > 1:
        row_grad[rows - 1] = math.nan
    valid, loss, grad = distill_definition(torch, z, index, value, t, row_grad, dtype)
    with handle(torch, "distill", dtype, rows, vocab, 0, top_k) as h:
        status = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
        got = h.distill(z, index, value, t, status=status)
        within(got, *loss, "loss")
        assert bool((status == 0).all())
        got, got_grad = h.distill_grad(z, index, value, row_grad, t)
        within(got, *loss, "loss with gradient")
        within(got_grad, *grad, "grad_logits")
        _, same = h.distill_grad(z, index, value, row_grad, t, grad_logits=z)      # in place
        assert same is z and torch.equal(z, got_grad)


def test_distillation_rows_without_a_softmax(torch):
    inf = math.inf
    z = torch.randn((6, 100), device="cuda")
    index = torch.arange(4, dtype=torch.int32, device="cuda").repeat(6, 1)
    value = torch.zeros((6, 4), device="cuda")
    index[1, 2] = 100                                       # outside
    index[2, 0] = -2                                        # outside
    value[3] = -inf                                         # the teacher's entries are all -infinity
    z[4] = -inf                                             # the student's logits are
    z[5, :50] = -inf                                        # half of them: a vocabulary of which a part is masked
    index[5] += 60
    value[5, 3] = -inf                                      # an entry of probability 0
    row_grad = torch.ones(6, device="cuda")
    with handle(torch, "distill", "f32", 6, 100, 0, 4) as h:
        status = torch.full((6,), -9, dtype=torch.int32, device="cuda")
        loss, grad = h.distill_grad(z, index, value, row_grad, status=status)
    assert status.tolist() == [0, 1, 1, 1, 1, 0]
    assert bool((loss[1:5] == 0).all()) and bool((grad[1:5] == 0).all())
    for r in (0, 5):
        valid, want, want_grad = distill_definition(torch, z[r:r + 1], index[r:r + 1], value[r:r + 1], 1.0, row_grad[:1], "f32")
        within(loss[r:r + 1], *want, "loss")
        within(grad[r:r + 1], *want_grad, "grad_logits")


def test_distillation_gradient_against_differences(torch):
    g = generator(torch, 21)
    z = torch.randn((3, 40), generator=g, device="cuda")
    index = torch.stack([torch.randperm(40, generator=g, device="cuda")[:6] for _ in range(3)]).int()
    value = torch.randn((3, 6), generator=g, device="cuda")
    row_grad = torch.rand(3, generator=g, device="cuda")
    with handle(torch, "distill", "f32", 3, 40, 0, 6) as h:
        grad = h.distill_grad(z, index, value, row_grad, 2.0)[1]
        for _ in range(4):
            by, eps = torch.randn((3, 40), generator=g, device="cuda"), 5e-2
            f = lambda s: float((h.distill(z + s * by, index, value, 2.0).double() * row_grad.double()).sum())  # noqa: E731
            diff = (8 * (f(eps) - f(-eps)) - (f(2 * eps) - f(-2 * eps))) / (12 * eps)
            slope = float((grad * by).double().sum())
            assert abs(diff - slope) <= 1e-3 * (1 + abs(slope))


# ---- the manner of the calls ----------------------------------------------------------------

def test_calls_replayed_from_a_graph(torch):
    """Each replay, with new inputs in the same buffers and eager work in between, against the same calls made
    outside the graph."""
    rows, vocab, hidden, k = 200, 3000, 96, 8
    h, w, labels, row_grad = head_inputs(torch, 31, rows, vocab, hidden, 0, 0, 0.2, "bf16")
    g = generator(torch, 32)
    z = (torch.randn((rows, vocab), generator=g, device="cuda") * 2).bfloat16()
    index = torch.stack([torch.randperm(vocab, generator=g, device="cuda")[:k] for _ in range(rows)]).int()
    value = torch.randn((rows, k), generator=g, device="cuda")
    from paper_2503_16815_amd import ends
    with ends.DeftEnds(ends.OPERATORS, torch.bfloat16, rows, vocab, hidden, k) as e:
        def calls():
            x = e.embed(labels, w, 2.0)
            loss, lse = e.head_loss(h, w, labels)
            gh, gw = e.head_grad(h, w, labels, lse, row_grad)
            e.embed_grad(labels, gh, grad_table=gw, accumulate=True)
            d, gz = e.distill_grad(z, index, value, row_grad, 2.0)
            return x, loss, lse, gh, gw, d, gz
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            calls()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            outs = calls()
        for rep in range(3):
            new = head_inputs(torch, 40 + rep, rows, vocab, hidden, 0, 0, 0.3 * rep, "bf16")
            for to, x in zip((h, w, labels, row_grad), new):
                to.copy_(x)
            z.copy_((torch.randn((rows, vocab), generator=g, device="cuda") * 2).bfloat16())
            want = [x.clone() for x in calls()]
            for x in outs:
                x.fill_(-7)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(outs, want):
                assert torch.equal(a, b)


def test_calls_on_two_streams(torch):
    """Two handles on two streams share nothing."""
    sets = [head_inputs(torch, 50 + i, 130, 2000, 64, 0, 0, 0.1, "bf16") for i in range(2)]
    from paper_2503_16815_amd import ends
    streams = [torch.cuda.Stream() for _ in range(2)]
    handles = [ends.DeftEnds(("head_loss", "head_grad"), torch.bfloat16, 130, 2000, 64) for _ in range(2)]
    def step(i, stream):
        h, w, labels, row_grad = sets[i]
        loss, lse = handles[i].head_loss(h, w, labels, stream=stream)
        return (loss, lse) + handles[i].head_grad(h, w, labels, lse, row_grad, stream=stream)
    want = [step(i, None) for i in range(2)]
    torch.cuda.synchronize()
    got = [[step(i, s) for i, s in enumerate(streams)] for _ in range(3)]
    torch.cuda.synchronize()
    for r in got:
        for i in range(2):
            assert all(torch.equal(a, b) for a, b in zip(r[i], want[i]))
    for e in handles:
        e.close()


def test_refusals(torch):
    from paper_2503_16815_amd import ends
    from paper_2503_16815_amd.binding import DEFT_ERR_INVALID_ARG, DEFT_ERR_LIMIT, DeftError
    bf = torch.bfloat16
    with ends.DeftEnds(("embed", "head_loss", "distill"), bf, 8, 100, 64, 4) as e:
        tok = torch.zeros(8, dtype=torch.int32, device="cuda")
        w = torch.zeros((100, 64), dtype=bf, device="cuda")
        h = torch.zeros((8, 64), dtype=bf, device="cuda")
        def code(f, *a, **k):
            with pytest.raises(DeftError) as err:
                f(*a, **k)
            return err.value.code
        assert code(e.embed_grad, tok, h, vocab=100) == DEFT_ERR_LIMIT                   # not served
        assert code(e.head_grad, h, w, tok, tok.float(), tok.float()) == DEFT_ERR_LIMIT
        nine = torch.zeros(9, dtype=torch.int32, device="cuda")
        assert code(e.embed, nine, w) == DEFT_ERR_LIMIT                                    # more rows than the handle's
        assert code(e.embed, tok, torch.zeros((101, 64), dtype=bf, device="cuda")) == DEFT_ERR_LIMIT
        assert code(e.embed, tok, torch.zeros((100, 65), dtype=bf, device="cuda")) == DEFT_ERR_LIMIT
        z = torch.zeros((8, 100), dtype=bf, device="cuda")
        idx, val = torch.zeros((8, 5), dtype=torch.int32, device="cuda"), torch.zeros((8, 5), device="cuda")
        assert code(e.distill, z, idx, val) == DEFT_ERR_LIMIT
        i4, v4 = idx[:, :4].contiguous(), val[:, :4].contiguous()
        for t in (0.0, -1.0, math.inf, math.nan):
            assert code(e.distill, z, i4, v4, t) == DEFT_ERR_INVALID_ARG
        for bad in (lambda: e.embed(tok.long(), w), lambda: e.embed(tok, w.float()), lambda: e.embed(tok.cpu(), w),
                    lambda: e.embed(tok, w.t()), lambda: e.embed(tok, w[0]), lambda: e.embed(tok[::2], w),
                    lambda: e.head_loss(h, w[:, :32], tok), lambda: e.head_loss(h, w, tok[:7]),
                    lambda: e.distill(z, i4, v4[:, :3]), lambda: e.distill(z, i4, v4.double()),
                    lambda: e.embed(tok, w, out=h[:7]), lambda: e.embed(tok, w, out=h.float()),
                    lambda: e.embed(tok, w, out=torch.zeros((1, 64), dtype=bf, device="cuda").expand(8, 64)),
                    lambda: e.distill_grad(z, i4, v4, torch.zeros(7, device="cuda"))):
            with pytest.raises(ValueError):
                bad()
        e.close()
        with pytest.raises(ValueError):
            e.embed(tok, w)
    with pytest.raises(DeftError) as err:
        ends.DeftEnds("embed", bf, 0, 1, 1)
    assert err.value.code == DEFT_ERR_INVALID_ARG
    with pytest.raises(DeftError) as err:                                                  # a type of table out of all proportion
        ends.DeftEnds(("head_loss", "head_grad"), torch.float32, 1 << 20, 1 << 21, 16384)
    assert err.value.code == 4
