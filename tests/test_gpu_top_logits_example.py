"""The example that trains on stored top logits: it runs, and the draft learns."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_draft_learns(capsys):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("train_on_top_logits",
                                                  os.path.join(ROOT, "examples", "train_on_top_logits.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    losses = m.main(["--steps", "20", "--batch", "2", "--positions", "24", "--vocab", "4001", "--top", "32"])
    assert len(losses) == 20 and all(math.isfinite(x) for x in losses)
    assert losses[-1] < 0.7 * losses[0]
    assert "acceptance" in capsys.readouterr().out
