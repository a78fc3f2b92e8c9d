"""Answers that the head drafts and the protected network's probabilities verify."""
import pytest

from _gpu import ct

pytestmark = pytest.mark.gpu


def test_answers_drawn_at_small_temperatures():
    """Drafts come from the distribution that they are verified by: logits 1e-7 apart at a temperature of 1e-8 leave e^-10 for the lesser."""
    import torch
    ct()
    from paper_2609_16742_gb300 import answer_head
    x = torch.tensor([0.0, 1e-7], device="cuda").repeat(4000, 1)
    answers, stood = answer_head.draw_answers(x, x, seed=1, temperature=torch.full((4000,), 1e-8, device="cuda"))
    # 4000 e^-10 = 0.18 expected: more than 8 have a probability below 1e-11
    assert stood.all() and int((answers == 0).sum()) <= 8
