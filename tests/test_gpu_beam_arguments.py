"""Arguments of a selection that raise errors of their own."""
import pytest
import torch

from paper_2609_34645_b200 import logits as L

pytestmark = pytest.mark.gpu


def test_settle_without_a_truth_value():
    x, score = torch.zeros(4, 100, device="cuda"), torch.zeros(4, device="cuda")
    for settle in (torch.zeros(2), torch.ones(3, device="cuda")):
        with pytest.raises(RuntimeError, match="ambiguous"):
            L.beam_select(x, score, 2, beams=2, settle=settle)
    plain, settled = L.beam_select(x, score, 2, beams=2), L.beam_select(x, score, 2, beams=2, settle=torch.ones(()))
    assert plain[1].tolist() == [[0, 0], [2, 2]] and settled[1].tolist() == [[0, 0], [2, 2]] and settled[2].tolist() == [[0, 1], [0, 1]]
