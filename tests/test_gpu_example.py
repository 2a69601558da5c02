"""The example runs its three stages together: every update lowers the loss on its own positions, and the answers keep to
the grammar and the vocabulary."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_post_training_step():
    spec = importlib.util.spec_from_file_location("post_training_step", os.path.join(ROOT, "examples", "post_training_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses, history, mask, which = m.main()
    assert all(after < before for before, after in losses)
    answers = history[:, m.PROMPT:]
    assert ((answers >= 0) & (answers < m.VOCAB)).all()
    assert (answers[which == 0] % 3 > 0).all()
