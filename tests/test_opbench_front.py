"""What opbench.py times of the embedding pair, the query and key norms and the orthogonalised update, and the bytes and operations it counts."""
import re

import pytest

from test_opbench import run

pytestmark = pytest.mark.gpu


def rate(out, name):
    ms, r = map(float, re.search(name + r".*?: ([\d.]+) ms ([\d.]+)", out).groups())
    return ms, r


@pytest.mark.parametrize("args,size", [([], 2), (["--f32"], 4), (["--f32", "--add"], 8), (["--add"], 4)])
def test_embedding(monkeypatch, capsys, args, size):
    T, V, d = 4096, 32768, 1024
    out = run(monkeypatch, capsys, "embed", "--m", str(T), "--n", str(V), "--k", str(d), *args)
    for name, want in (("embed fwd", 6 * T * d), ("embed bwd", 4 * T * d + size * V * d)):
        ms, r = rate(out, name)
        assert abs(ms * r * 1e6 - want) <= 0.02 * want, (name, out)      # as far as the printed digits go


@pytest.mark.parametrize("kv", [0, 4])
def test_query_and_key_norms(monkeypatch, capsys, kv):
    T, h, dh = 4 * 1024, 16, 128
    out = run(monkeypatch, capsys, "qk", "--batch", "4", "--seq", "1024", "--heads", str(h), "--kv-heads", str(kv), "--dh", str(dh))
    kv = kv or h
    for name, want in (("qk fwd", 4 * T * (h + 2 * kv) * dh), ("qk bwd", 6 * T * (h + kv) * dh + 4 * T * kv * dh)):
        ms, r = rate(out, name)
        assert abs(ms * r * 1e6 - want) <= 0.02 * want, (name, out)


@pytest.mark.parametrize("args", [[], ["--f32", "--momentum"]])
def test_orthogonalised_update(monkeypatch, capsys, args):
    import opbench
    real, seen = opbench.ppu.ppu_orthogonalize, []
    monkeypatch.setattr(opbench.ppu, "ppu_orthogonalize", lambda G, **kw: seen.append((G.dtype, kw["momentum"] is not None)) or real(G, **kw))
    out = run(monkeypatch, capsys, "ortho", "--batch", "3", "--m", "512", "--k", "1536", *args)
    ms, r = rate(out, "ortho 3 x 512 x 1536")
    want = 5 * 3 * 512 ** 2 * (3 * 1536 + 512)
    assert abs(ms * r * 1e9 - want) <= 0.02 * want and set(seen) == {(opbench.torch.float32 if args else opbench.torch.bfloat16, bool(args))}
