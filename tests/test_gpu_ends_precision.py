"""What 32 bits are worth: the head's sums hold 24 bits, distillation's probabilities do whatever a row's logits have in
common.

Head (u = 2^-24): operands are taken apart exactly and the products left out are 2^-21 of the others at most.  A sum
of K products is rounded some 6 K / 8 times, each time by less than u of what is summed so far, in no preferred direction: 23 u / 2 of the norm
for K = 700, 0.7e-6.  The logits' errors and the exponentials' (arguments of about 10: 10 u in all) come into d in
proportion, 0.6e-6 each.  Together 1.5e-6 for losses and twice that, 3e-6, for the gradients, which sum twice.  A single one of the
six products left out costs 3e-6 or more of the losses and 1e-5 of the gradients (worked out on the CPU for these inputs).

Distillation: with a = (z - largest) / T an exponential is off by 6 u |a| (difference, two constants, product) and 4 u, a
sum of them by the mean of that and 200 u (chains of up to 200 additions); likewise the teacher's with b."""
import pytest

from tests.test_gpu_ends import generator, handle, head_definition, head_inputs, torch, within  # noqa: F401 (torch is a fixture)

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


@pytest.mark.parametrize("rows,vocab,hidden", [(1, 700, 96), (64, 700, 96), (100, 700, 96), (300, 650, 640), (65, 600, 700)])
def test_head_in_32_bits(torch, rows, vocab, hidden):  # noqa: F811
    h, w, labels, row_grad = head_inputs(torch, rows + hidden, rows, vocab, hidden, 0, 0, 0.0, "f32")
    _, loss, lse, gh, gw = head_definition(torch, h, w, labels, 1.0, row_grad, "f32")
    with handle(torch, ("head_loss", "head_grad"), "f32", rows, vocab, hidden) as e:
        got_loss, got_lse = e.head_loss(h, w, labels)
        got_gh, got_gw = e.head_grad(h, w, labels, got_lse, row_grad)
    off = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert off(got_lse, lse[0]) <= 1.5e-6 and off(got_loss, loss[0]) <= 1.5e-6
    assert off(got_gh, gh[0]) <= 3e-6 and off(got_gw, gw[0]) <= 3e-6


@pytest.mark.parametrize("rows,vocab,top_k,t", [(5, 50257, 32, 2.0), (4, 4097, 17, 1.0), (300, 1000, 64, 3.0), (3, 70001, 100, 0.7), (2, 131073, 600, 2.0)])
@pytest.mark.parametrize("offset", [0.0, 4000.0, -30000.0])
def test_distillation_in_32_bits(torch, rows, vocab, top_k, t, offset):  # noqa: F811
    g = generator(torch, rows + vocab)
    z = torch.randn((rows, vocab), generator=g, device="cuda") * 2.5 + offset
    index = torch.stack([torch.randperm(vocab, generator=g, device="cuda")[:top_k] for _ in range(rows)]).int()
    value = torch.randn((rows, top_k), generator=g, device="cuda") * 3 + offset
    row_grad = torch.rand(rows, generator=g, device="cuda") + 0.5
    with handle(torch, "distill", "f32", rows, vocab, 0, top_k) as e:
        alone = e.distill(z, index, value, t)
        loss, grad = e.distill_grad(z, index, value, row_grad, t)
    a = (z.double() - z.double().amax(1, keepdim=True)) / t
    b = (value.double() - value.double().amax(1, keepdim=True)) / t
    log_q, log_p = torch.log_softmax(a, 1), torch.log_softmax(b, 1)
    q, p, at = log_q.exp(), log_p.exp(), index.long()
    rel_q = E * (6 * (a.abs() + (q * a.abs()).sum(1, keepdim=True)) + 220)
    rel_p = E * (6 * (b.abs() + (p * b.abs()).sum(1, keepdim=True)) + 220)
    lq, aq = log_q.gather(1, at), a.abs().gather(1, at)
    want = (p * (log_p - lq)).sum(1) * t * t
    size = (p * (rel_p * (log_p - lq).abs() + E * (6 * (aq + b.abs()) + 460 + 2 * log_p.abs() + 2 * lq.abs()))).sum(1)
    within(alone, want, t * t * size, "loss")
    within(loss, want, t * t * size, "loss with gradient")
    by = row_grad.double()[:, None] * t
    d = q.scatter_add(1, at, -p) * by
    err = by * ((q * rel_q).scatter_add(1, at, p * rel_p) + 4 * E * q.scatter_add(1, at, p)) + 1e-37
    within(grad, d, err, "grad_logits")
