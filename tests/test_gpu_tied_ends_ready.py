"""When the pieces of the shared table's gradient are final: behind the last part that is added to them."""
import json

import pytest

pytestmark = pytest.mark.gpu


def test_pieces_are_ready_when_nothing_is_added_any_more(capsys):
    from paper_2503_16815_amd import tied_ends
    assert tied_ends.main(["--rows", "8192", "--vocab", "60000", "--hidden", "256", "--steps", "3"]) == 0
    said = json.loads(capsys.readouterr().out)
    head, ready = said["head_part_us"], said["pieces_ready_us"]
    assert len(head) == len(ready) > 1
    assert head == sorted(head) and head[0] > 0.0
    # the distilled positions' part and the embedding's come behind the head's, into every piece
    assert min(ready) > max(head) and max(ready) <= said["backward_us"]
    # the first window that a bucket can be sent in is the next iteration's forward pass
    assert said["windows"] == [max(1, int(t / 10)) for t in (said["forward_us"], said["backward_us"])] * 2
