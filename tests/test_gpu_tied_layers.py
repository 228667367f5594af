"""The step with feed-forward blocks between its ends: the layers' gradients as a program uses them, against torch's automatic
differentiation of the same step in 64 bits, delayed merges, the buckets' schedule, and the program itself."""
import json

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _step(dtype, save, layers=2, rows=150, vocab=1300, hidden=48, inner=80):
    import torch
    from paper_2503_16815_amd import tied_ends
    step = tied_ends.Step.create(rows, vocab, hidden, dtype=dtype, top_k=4, layers=layers, inner=inner, save=save)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    tokens = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    tokens[5] = -1
    labels = torch.roll(tokens, -1)
    labels[-1] = -1
    row_grad = torch.rand(rows, generator=g, device="cuda")
    leaves = [step.table, step.mix, *[w for layer in step.layers for w in layer]]
    leaves = [w.double().requires_grad_() for w in leaves]
    table, mix = leaves[:2]
    x = torch.where((tokens >= 0)[:, None], table[tokens.long().clamp(min=0)], 0.0) * step.scale
    h = torch.tanh(x @ mix)
    for i in range(layers):
        wg, wu, wd = leaves[2 + 3 * i:5 + 3 * i]
        h = h + (torch.nn.functional.silu(h @ wg.T) * (h @ wu.T)) @ wd.T
    logp = torch.log_softmax(h @ table.T, dim=1)
    per = torch.where(labels >= 0, -logp.gather(1, labels.long().clamp(min=0)[:, None]).squeeze(1), 0.0)
    (per * row_grad.double()).sum().backward()
    return step, tokens, labels, row_grad, per.detach(), [w.grad for w in leaves]


# 32 bits: sums a few hundred terms deep, a part in 1e4 of the norm.  In 8 bits an element is off by at most (1 + 2^-7) / 254 of the
# largest of its 32, so a group by at most sqrt(32) / 252 = 0.0225 of its norm: a layer's gradients have three such factors (its
# input and both projections, whose activations have slopes below 1.13), and each layer passes its part on.
@pytest.mark.parametrize("save,limit", [(None, 1e-4), ("full", 1e-4), ("packed", 2 * 3 * 1.13 * 0.0225)])
def test_step_against_automatic_differentiation(save, limit):
    import torch
    step, tokens, labels, row_grad, per, grads = _step(torch.float32, save)
    x, h, loss, lse = step.forward(tokens, labels)
    grad_table, grad_mix, _ = step.backward(tokens, labels, x, h, lse, row_grad)
    assert float((loss.double() - per).norm()) <= 1e-4 * float(per.norm())
    got = [grad_table, grad_mix, *[w for layer in step.grad_layers for w in layer]]
    for a, b in zip(got, grads):
        assert float((a.double() - b).norm()) <= limit * float(b.norm())
    # an update delayed by one iteration: both iterations' gradients in one buffer
    once = [t.clone() for t in got]
    step.backward(tokens, labels, x, h, lse, row_grad, merge=True)
    torch.cuda.synchronize()
    for a, b in zip(got[2:], once[2:]):
        assert float((a.double() - 2 * b.double()).norm()) <= 1e-5 * float(b.norm())
    step.ends.close()
    step.block.close()


def test_layers_buckets_are_scheduled(oracle):
    import torch
    from paper_2503_16815_amd import tied_ends
    step = tied_ends.Step.create(64, 1300, 48, dtype=torch.float32, layers=3, inner=80)
    kb, out = tied_ends.schedule(step, 300.0, 700.0, 2, 0.2)
    bare, _ = tied_ends.schedule(tied_ends.Step.create(64, 1300, 48, dtype=torch.float32), 300.0, 700.0, 2, 0.2)
    # each matrix, 80 x 48 x 4 bytes at 0.2 GB/s, takes 76.8 us: two buckets of 38 us, as a quarter of the window is 75
    assert kb.weights.shape[1] == bare.weights.shape[1] + 3 * 3 * 2
    assert kb.weights.max() <= 8 and (kb.weights[0, -18:] == 4).all()
    ref = oracle.solve_batch(kb, nthreads=1)
    for name in ("status", "total_value", "knap_value", "knap_load", "assignment"):
        assert np.array_equal(getattr(out, name).cpu().numpy(), getattr(ref, name)), name


def test_the_program_runs_with_layers(capsys):
    from paper_2503_16815_amd import tied_ends
    assert tied_ends.main(["--rows", "512", "--vocab", "9000", "--hidden", "256", "--steps", "3", "--layers", "2"]) == 0
    said = json.loads(capsys.readouterr().out)
    ready = said["layers_ready_us"]
    assert len(ready) == 2 and all(len(e) == 2 for e in ready)
    # the last layer's gradients are final first; w_down's before the others'
    order = [*ready[1], *ready[0]]
    assert order == sorted(order) and max(order) <= said["backward_us"] and max(said["head_part_us"]) <= min(order)
    assert len(said["window_of_bucket"]) == len(said["bucket_times"])
