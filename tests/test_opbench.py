"""What opbench.py times and counts."""
import re
import sys

import pytest

pytestmark = pytest.mark.gpu


def run(monkeypatch, capsys, *args):
    import opbench
    monkeypatch.setattr(sys, "argv", ["opbench.py", *args, "--iters", "2", "--warmup", "1"])
    opbench.main()
    return capsys.readouterr().out


def test_cross_entropy_is_called_with_a_target_made_beforehand(monkeypatch, capsys):
    import opbench
    real, seen = opbench.ppu.ppu_head_xent, []
    monkeypatch.setattr(opbench.ppu, "ppu_head_xent", lambda X, E, target, **kw: seen.append(target) or real(X, E, target, **kw))
    run(monkeypatch, capsys, "head", "--m", "64", "--n", "300", "--k", "64")
    assert len(seen) == 3 and all(t is seen[0] for t in seen)
