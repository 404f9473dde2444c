"""opbench.py embed --in-place: the table's gradient in the place of another one; the bytes it counts are dout and the rows with tokens, read and written."""
import pytest

from test_opbench import run
from test_opbench_front import rate

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("args,size", [(["--in-place"], 2), (["--in-place", "--f32"], 4)])
def test_gradient_in_place(monkeypatch, capsys, args, size):
    import opbench
    T, V, d = 4096, 32768, 1024
    real, seen = opbench.ppu.ppu_embed_bwd, []

    def call(ids, dout, V, **kw):
        out = real(ids, dout, V, **kw)
        seen.append((out is kw["add"] or out.data_ptr() == kw["add"].data_ptr(), ids.unique().numel()))
        return out
    monkeypatch.setattr(opbench.ppu, "ppu_embed_bwd", call)
    out = run(monkeypatch, capsys, "embed", "--m", str(T), "--n", str(V), "--k", str(d), *args)
    ms, r = rate(out, "embed bwd")
    want = 4 * T * d + 2 * size * seen[0][1] * d
    assert all(s[0] for s in seen) and abs(ms * r * 1e6 - want) <= 0.02 * want, out
