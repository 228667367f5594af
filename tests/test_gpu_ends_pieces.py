"""The events of the head's gradient, piece by piece of the vocabulary."""
import pytest

from tests.test_gpu_ends import head_inputs, torch  # noqa: F401 (torch is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("need_weight", [True, False])
def test_more_events_than_pieces(torch, need_weight):  # noqa: F811
    """An event is recorded once the rows below its bound are final: those whose bound lies past the vocabulary's end
    after the last piece, not before the first."""
    from paper_2503_16815_amd import ends
    rows, vocab, hidden = 2000, 5000, 512
    h, w, labels, row_grad = head_inputs(torch, 8, rows, vocab, hidden, 0, 0, 0.2, "bf16")
    with ends.DeftEnds(("head_loss", "head_grad"), h.dtype, 1 << 17, vocab, hidden) as e:
        pieces = -(-vocab // e.info().vocab_piece)
        assert pieces > 2
        lse = e.head_loss(h, w, labels)[1]
        for _ in range(2):
            events = [torch.cuda.Event(enable_timing=True) for _ in range(pieces + 3)]
            e.head_grad(h, w, labels, lse, row_grad, piece_events=events, need_weight=need_weight)
            torch.cuda.synchronize()
            at = [events[0].elapsed_time(x) for x in events[1:]]
            assert at == sorted(at) and at[0] > 0.0, at
