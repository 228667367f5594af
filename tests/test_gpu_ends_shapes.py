"""Operators by the variants that their sizes choose.  The head on sizes that run each shape of its products' tiles (256 x 256, 192 x 256, 160 x 256, 256 x 128,
128 x 128; 256 x 64 is what up to 64 positions run) in each of the four products, last tiles that pass the
operands' ends among them.  Definitions and bounds as in test_gpu_ends.py."""
import pytest

from tests.test_gpu_ends import (distill_definition, generator, handle, head_definition, head_inputs, matrix,  # noqa: F401
                                 torch, within)  # (torch is a fixture)

pytestmark = pytest.mark.gpu

SIZES = [  # rows, vocab, hidden: what the 16-bit types run there
    (777, 12297, 40),     # logits 256 x 256
    (520, 13625, 40),     # logits 192 x 256
    (520, 13069, 40),     # logits 160 x 256
    (777, 10369, 40),     # logits 192 x 256, the last tile passes the last panel of 256 columns
    (520, 13300, 40),     # logits 160 x 256, likewise
    (70, 2033, 40),       # logits 256 x 128
    (520, 10901, 320),    # weights' gradient 256 x 128
    (70, 13110, 777),     # weights' gradient 256 x 256
    (70, 9223, 1000),     # weights' gradient 192 x 256
    (70, 9352, 777),      # weights' gradient 160 x 256
    (1100, 8153, 130),    # hidden states' gradient 256 x 128, in 16 parts
    (520, 4044, 1601),    # hidden states' gradient 192 x 256, in 8 parts
    (520, 8150, 777),     # hidden states' gradient 160 x 256, in 16 parts
    (4096, 600, 1024),    # hidden states' gradient without parts
]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,vocab,hidden", SIZES)
def test_head_by_shape(torch, dtype, rows, vocab, hidden):  # noqa: F811
    h, w, labels, row_grad = head_inputs(torch, rows + hidden, rows, vocab, hidden, 0, 0, 0.05, dtype)
    valid, loss, lse, gh, gw = head_definition(torch, h, w, labels, 1.0, row_grad, dtype)
    with handle(torch, ("head_loss", "head_grad"), dtype, rows, vocab, hidden) as e:
        got_loss, got_lse = e.head_loss(h, w, labels)
        within(got_loss, *loss, "loss")
        within(got_lse, *lse, "lse")
        got_gh, got_gw = e.head_grad(h, w, labels, got_lse, row_grad)
        within(got_gh, *gh, "grad_hidden")
        within(got_gw, *gw, "grad_weight")
        again = e.head_grad(h, w, labels, got_lse, row_grad)
        assert torch.equal(again[0], got_gh) and torch.equal(again[1], got_gw)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows,vocab,hidden", [(15, 8339, 173), (64, 3000, 256), (300, 5000, 320)])
def test_roundings_of_the_derivative(torch, dtype, rows, vocab, hidden):  # noqa: F811
    """The hidden states' gradient is as close as its own type allows, a half more at most, and so is the weights'
    of up to 64 positions: rounding the derivative costs next to nothing there.  (The norm of a rounding of relative
    size up to u, evenly spread, is u / sqrt(3) at most.)"""
    h, w, labels, row_grad = head_inputs(torch, 9, rows, vocab, hidden, 0, 0, 0.0, dtype)
    _, _, _, gh, gw = head_definition(torch, h, w, labels, 1.0, row_grad, dtype)
    half = {"bf16": 2.0 ** -9, "f16": 2.0 ** -12}[dtype] * 2 / 3 ** 0.5
    with handle(torch, ("head_loss", "head_grad"), dtype, rows, vocab, hidden) as e:
        got = e.head_grad(h, w, labels, e.head_loss(h, w, labels)[1], row_grad)
    off = [float((g.double() - x[0]).norm() / x[0].norm()) for g, x in zip(got, (gh, gw))]
    assert off[0] <= 1.5 * half
    if rows <= 64:
        assert off[1] <= 1.5 * half


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_row_gradients_of_any_size(torch, dtype):  # noqa: F811
    """Each row's factor is taken apart exactly: rows of very small and very large factors, zeros among them, have
    gradients as exact as the others."""
    rows, vocab, hidden = 200, 700, 96
    h, w, labels, row_grad = head_inputs(torch, 77, rows, vocab, hidden, 0, 0, 0.0, dtype)
    top = 6 if dtype == "f16" else 30
    row_grad = row_grad * torch.pow(2.0, torch.randint(-top, top, (rows,), device="cuda").float())
    row_grad[::17] = 0.0
    row_grad[1::17] *= -1.0
    _, _, _, gh, gw = head_definition(torch, h, w, labels, 1.0, row_grad, dtype)
    with handle(torch, ("head_loss", "head_grad"), dtype, rows, vocab, hidden) as e:
        got_gh, got_gw = e.head_grad(h, w, labels, e.head_loss(h, w, labels)[1], row_grad)
        within(got_gh, *gh, "grad_hidden")
        assert bool((got_gh[::17] == 0).all())
        # (columns of the hidden states scaled below the largest factor's range add less than its rounding)
        floor = float(row_grad.abs().max()) * (2.0 ** -38 if dtype == "f16" else 0.0) * rows * float(h.abs().max())
        within(got_gw, gw[0], gw[1] + floor, "grad_weight")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,vocab,hidden,pad", [(300, 1001, 128, 0), (300, 1001, 128, 64), (520, 8150, 832, 0), (520, 4044, 1600, 64),
                                                   (70, 2033, 64, 64), (64, 517, 192, 0), (300, 1001, 100, 28)])
def test_what_lies_behind_the_table(torch, dtype, rows, vocab, hidden, pad):  # noqa: F811
    """Rows behind the table's last one and what lies between its rows are read by no product, whatever they hold."""
    h, w, labels, row_grad = head_inputs(torch, rows + vocab, rows, vocab, hidden, 0, 0, 0.05, dtype)
    _, _, _, gh, gw = head_definition(torch, h, w, labels, 1.0, row_grad, dtype)
    around = torch.full((vocab + 300, hidden + pad), float("nan"), dtype=w.dtype, device=w.device)
    around[:vocab, :hidden] = w
    inside = around[:vocab, :hidden]
    with handle(torch, ("head_loss", "head_grad"), dtype, rows, vocab, hidden) as e:
        loss, lse = e.head_loss(h, w, labels)
        plain = e.head_grad(h, w, labels, lse, row_grad)
        got_loss, got_lse = e.head_loss(h, inside, labels)
        got = e.head_grad(h, inside, labels, got_lse, row_grad)
        within(plain[0], *gh, "grad_hidden")
        within(plain[1], *gw, "grad_weight")
        for a, b in zip((loss, lse, *plain), (got_loss, got_lse, *got)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,vocab,top_k", [(2100, 1003, 8), (900, 12345, 20), (600, 30001, 8), (600, 50257, 33), (300, 70001, 600)])
def test_distillation_from_row_to_row(torch, dtype, rows, vocab, top_k):  # noqa: F811
    """More rows than workgroups run at once, so that each goes on from row to row; rows without an entry among them."""
    g = generator(torch, rows + vocab)
    z = matrix(torch, g, rows, vocab, dtype, 2.5, 1, 0)
    index = torch.rand((rows, 4 * top_k), generator=g, device="cuda").argsort(1)[:, :top_k].int() * (vocab // (4 * top_k))
    value = torch.randn((rows, top_k), generator=g, device="cuda") * 3
    index[torch.rand((rows, top_k), generator=g, device="cuda") < 0.2] = -1
    index[3::7] = -1
    z[3::7] = float("nan")
    row_grad = torch.rand(rows, generator=g, device="cuda") * 2
    valid, loss, grad = distill_definition(torch, z, index, value, 2.0, row_grad, dtype)
    with handle(torch, "distill", dtype, rows, vocab, 0, top_k) as e:
        within(e.distill(z, index, value, 2.0), *loss, "loss")
        got, got_grad = e.distill_grad(z, index, value, row_grad, 2.0)
        within(got, *loss, "loss with gradient")
        within(got_grad, *grad, "grad_logits")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("factor", [1.02, 1.4, 1.98])
def test_roundings_where_all_rows_count_alike(torch, dtype, factor):  # noqa: F811
    """The weights' gradient of a mean: the labels' entries are rounded just below a power of two, whatever the mean's
    factor.  (In the norm, with h the largest relative rounding / sqrt(3): the output's own 0.74 h, mantissas spread
    evenly by their logarithm; the labels' entries 0.5 h / 0.9 for probabilities below 0.1; together 0.92 h, and a
    seventh more at most.)"""
    rows, vocab, hidden = 700, 9001, 320
    h, w, labels, _ = head_inputs(torch, 21, rows, vocab, hidden, 0, 0, 0.0, dtype)
    h = (h * 0.25).to(h.dtype)
    row_grad = torch.full((rows,), factor / 4, device="cuda")
    _, _, _, _, gw = head_definition(torch, h, w, labels, 1.0, row_grad, dtype)
    at_most = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}[dtype] / 3 ** 0.5
    with handle(torch, ("head_loss", "head_grad"), dtype, rows, vocab, hidden) as e:
        lse = e.head_loss(h, w, labels)[1]
        z = (h.double() * w[labels.long()].double()).sum(1)
        assert float((z - lse.double()).exp().max()) < 0.1
        got = e.head_grad(h, w, labels, lse, row_grad)[1]
    assert float((got.double() - gw[0]).norm() / gw[0].norm()) <= 1.05 * at_most


@pytest.mark.parametrize("rows", [1, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("vocab,hidden,pad,shift", [(1, 1, 0, 0), (127, 15, 1, 1), (129, 63, 0, 1), (1000, 64, 3, 0), (4099, 131, 0, 0), (300, 1600, 2, 3)])
def test_few_logits_in_32_bits(torch, rows, vocab, hidden, pad, shift):  # noqa: F811
    """The loss of up to 64 positions at the edges of its tiles; what lies between and behind the rows is never read."""
    h, w, labels, row_grad = head_inputs(torch, rows * 7 + vocab, rows, vocab, hidden, pad, shift, 0.0, "f32")
    if rows > 2:
        labels[1] = -1
    valid, loss, lse, _, _ = head_definition(torch, h, w, labels, 0.7, row_grad, "f32")
    around = torch.full((vocab + 200, hidden + 5), float("nan"), device="cuda")
    around[:vocab, :hidden] = w
    h[~valid] = float("nan")
    with handle(torch, ("head_loss",), "f32", rows, vocab, hidden) as e:
        got = e.head_loss(h, around[:vocab, :hidden], labels, 0.7)
        within(got[0], *loss, "loss")
        within(got[1], *lse, "lse")
