"""Forms and ranges of the head losses beside those of test_head_loss.py, by the same definition in 64 bits
and the same count of roundings."""
import numpy as np
import pytest

from test_head_loss import bf16, definition, hard

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("T,V", [(256, 2048), (24, 33000)])      # one warp to a row, several
def test_powers_beyond_the_common_reference_are_rounded_once(T, V):
    """Logits 50 to 80 nats from 0, the pieces' largest ones different: every piece has a reference of its own.  Column c > 1 of E
    is 1 for one id and 0 elsewhere, and X is 0 but for its first two columns: dX[t, c] = w p of one id, its
    power rounded to bf16 and the result rounded once.  The row's factor is taken out by the row's mean.  A rounding to nearest bf16 has a relative error of rms 2^-7 / sqrt 12 times the rms of 1 / m
    over mantissas m in [1, 2) (log-uniform: sqrt(3 / 8 / ln 2)), 1.66e-3: two make 2.35e-3, three 2.87e-3."""
    import torch
    from paper_2509_22418_b200 import ppu
    d = 128
    rng = np.random.default_rng(V)
    E = np.zeros((V, d))
    E[:, 0], E[:, 1] = 1.0, 3.0 * rng.standard_normal(V)
    at = rng.permutation(V)[: d - 2]
    E[at, np.arange(2, d)] = 1.0
    Et, E = bf16(E)
    x = np.zeros((T, d))
    x[:, 0], x[:, 1] = 65.0, rng.uniform(0.9, 1.1, T)
    Xt, X = bf16(x)
    pieces = np.array([(X @ E[a : a + 64].T).max(1) for a in range(0, V, 64)])
    assert pieces.min() > 60 * np.log(2) and (pieces == pieces.max(0)).mean() < 0.1
    target = rng.choice(np.setdiff1d(np.arange(V), at), T).astype(np.int32)
    ids, q, ent, _ = hard(target)
    w = np.ones(T)
    R = definition(X, E, ids, q, ent, w, 1.0)
    got = ppu.ppu_head_xent(Xt.cuda(), Et.cuda(), torch.from_numpy(target).cuda(), row_weight=torch.ones(T, device="cuda"))
    rel = got[3].double().cpu().numpy()[:, 2:] / R["dX"][:, 2:] - 1
    assert np.abs(rel).max() <= 3 * 2.0 ** -8 * (1 + 2.0 ** -7) + 2.0 ** -12     # power, factor, result: half a step each; the logits 16 2^-23 80
    rel -= rel.mean(1, keepdims=True)
    one = 2.0 ** -7 / np.sqrt(12) * np.sqrt(3 / 8 / np.log(2))
    assert np.sqrt((rel ** 2).mean()) <= one * (np.sqrt(2) + np.sqrt(3)) / 2


# ---- refusals, on the host ----------------------------------------------------------------------
def test_gradients_are_named_exactly():
    """A word that is none of those documented is refused, whatever letters it has."""
    import torch
    from paper_2509_22418_b200 import ppu
    X, E, t = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(32, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    for word in ("none", "both", "X", "", "x,e", "ee"):
        for call in (lambda: ppu.ppu_head_xent(X, E, t, grad=word), lambda: ppu.ppu_head_distill(X, E, t[:, None], X[:, :1].float(), grad=word)):
            with pytest.raises(ppu.PpuError, match="grad"):
                call()
    assert [ppu._grads(g) for g in (True, False, "x", "e", "xe", "ex", None)] == [3, 0, 1, 2, 3, 3, 0]


def test_sizes_that_do_not_fit_are_refused():
    """Sizes beyond 32 bits: not the workspace of what is left of them."""
    from paper_2509_22418_b200 import ppu
    for big in (2 ** 31, 2 ** 32 + 8, -2 ** 32 + 8, 2 ** 64 + 8):
        for at in range(3):
            sizes = [8, 64, 100]
            sizes[at] = big
            with pytest.raises(ppu.PpuError) as e:
                ppu.ppu_head_query_bytes(*sizes)
            assert e.value.code == -2
        for kw in (dict(grads=big), dict(chunk_rows=big), dict(k=big)):
            with pytest.raises(ppu.PpuError):
                ppu.ppu_head_query_bytes(8, 64, 100, **kw)
        for sizes in ((big, 64), (8, big), (8, 64, big)):
            with pytest.raises(ppu.PpuError):
                ppu.ppu_norm_gate_query_bytes(*sizes)
