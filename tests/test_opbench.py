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


@pytest.mark.parametrize("rows", [0, 1])
def test_bytes_of_the_norm_pair_hold_the_gate(monkeypatch, capsys, rows):
    T, d = 8192, 2048
    out = run(monkeypatch, capsys, "norm", "--m", str(T), "--k", str(d), "--gate-rows", str(rows))
    gate = 4 * d * (T if rows else 1)
    for name, want in (("fwd", 12 * T * d + gate), ("bwd", 18 * T * d + 2 * gate)):      # read forward; read, and its gradient written
        ms, rate = map(float, re.search(name + r".*: ([\d.]+) ms (\d+) GB/s", out).groups())
        assert abs(ms * rate * 1e6 - want) <= 0.01 * want, (name, out)      # as far as the printed digits go


@pytest.mark.parametrize("args,want", [([], "xe"), (["--grad", "x"], "x"), (["--grad", "none"], False), (["--no-grad"], False)])
def test_gradients_of_the_head(monkeypatch, capsys, args, want):
    import opbench
    real, seen = opbench.ppu.ppu_head_xent, []
    monkeypatch.setattr(opbench.ppu, "ppu_head_xent", lambda *a, grad, **kw: seen.append(grad) or real(*a, grad=grad, **kw))
    out = run(monkeypatch, capsys, "head", "--m", "64", "--n", "300", "--k", "64", *args)
    assert seen == [want] * 3 and f"grad={want or 'none'} " in out
