"""Losses of hidden states against the vocabulary (ppu_head_xent, ppu_head_distill) against their
definition in 64 bits, element by element, with tolerances derived from the operations' roundings.

Roundings counted (u = 2^-24 for fp32, half a step; bf16 half a step 2^-8):
  a logit: products of bf16 are exact in fp32; the tensor cores add 16 at a time to an fp32 sum, each
    addition off by at most a whole step 2^-23 of the sum of magnitudes: (d / 16 + 8) 2^-23 sum |x e|;
  log-sum-exp: the largest logit error, the exponentials' relative error (2^-21 with the rounding of their
    argument: |argument| u / ln 2 more) and the rounding of the result;
  ds = f u: the stored power u is bf16, and the row's factor is moved by up to half a bf16 step so that the
    entries' places round well: 2 * 2^-8 of Q p |w| (an entry's place: 2^-8 of its own value), beside the
    logits' errors; for dE the factor is multiplied into X, which is rounded to bf16 again: 2^-8 |ds| more;
  dX, dE: the errors of ds times the other operand's magnitudes, the sums' (n / 16 + 8) 2^-23 of the sum of
    magnitudes, and the result's own half step.
"""
import ctypes as C
import math

import numpy as np
import pytest

gpu = pytest.mark.gpu
U = 2.0 ** -24
BF = 2.0 ** -8


def bf16(a):
    import torch
    t = torch.from_numpy(np.asarray(a, dtype=np.float32)).bfloat16()
    return t, t.double().numpy()


def definition(X, E, ids, q, entropy, w, temp):
    """ids, q [T, k] (q = 0 where absent): losses, lse, ds, and dX, dE."""
    s = X @ E.T / temp
    m = s.max(1, keepdims=True)
    lse = m[:, 0] + np.log(np.exp(s - m).sum(1))
    T = len(X)
    row = entropy + (q * (lse[:, None] - s[np.arange(T)[:, None], ids])).sum(1)
    Q = q.sum(1)
    p = np.exp(s - lse[:, None])
    ds = Q[:, None] * p
    np.add.at(ds, (np.arange(T)[:, None], ids), -q)
    ds *= w[:, None]
    return dict(s=s, lse=lse, row=row, loss=(w * row).sum(), p=p, Q=Q, ds=ds, dX=ds @ E / temp, dE=ds.T @ X / temp)


def tolerances(X, E, q, w, temp, R, entropy):
    d, T, V = X.shape[1], len(X), len(E)
    mag = (np.abs(X) @ np.abs(E).T) / temp
    s_err = (d / 16 + 8) * 2 * U * mag + 2 * U * np.abs(R["s"])
    worst = s_err.max(1)
    spread = np.abs(R["s"]).max(1) + np.abs(R["lse"])
    lse = worst + 2.0 ** -21 + 4 * U * spread + 8 * U
    row = R["Q"] * (lse + worst) + 32 * U * (np.abs(entropy) + (np.abs(q).sum(1)) * (spread + 8))
    both = (s_err + lse[:, None]) * 1.01
    ds = np.abs(w)[:, None] * R["Q"][:, None] * R["p"] * (2 * BF + 2.0 ** -14 + both) + BF * np.abs(R["ds"]) + np.abs(w)[:, None] * 64 * U
    ds_e = ds * (1 + BF) + BF * np.abs(R["ds"])
    # (64 U: the entries' own places, 1 - p formed from q and p in fp32)
    sums = lambda n: (n / 16 + 12) * 2 * U  # noqa: E731
    dX = ds @ np.abs(E) / temp + sums(V) * (np.abs(R["ds"]) @ np.abs(E)) / temp
    dE = ds_e.T @ np.abs(X) / temp + sums(T) * (np.abs(R["ds"]).T @ np.abs(X)) / temp
    tiny = 1e-30
    return dict(lse=lse, row=row, loss=(np.abs(w) * row).sum() + 64 * U * (np.abs(w * R["row"])).sum() + tiny,
                dX=dX * (1 + BF) + BF * np.abs(R["dX"]) + tiny, dE=dE * (1 + BF) + BF * np.abs(R["dE"]) + tiny)


def check(got, R, tol):
    names = ("loss", "row", "lse", "dX", "dE")
    for n, g in zip(names, got):
        if g is None:
            continue
        g = g.detach().float().cpu().numpy().astype(np.float64)
        err = np.abs(g - R[n])
        assert np.all(err <= tol[n]), (n, float(err.max()), float((err / tol[n]).max()))


def make(T, d, V, seed, spread=3.0, raise_target=0.8):
    rng = np.random.default_rng(seed)
    Et, E = bf16(rng.standard_normal((V, d)) * (spread / math.sqrt(d)))
    target = rng.integers(0, V, T).astype(np.int32)
    # the ends of the vocabulary and of the pieces it is worked in are among the targets
    edge = [v for v in (0, 63, 64, V - 1, V - 2) if 0 <= v < V]
    target[: min(T, len(edge))] = edge[: min(T, len(edge))]
    Xt, X = bf16(rng.standard_normal((T, d)) + raise_target * E[target])
    return rng, Xt.cuda(), X, Et.cuda(), E, target


def hard(target):
    there = target >= 0
    return np.maximum(target, 0)[:, None].astype(np.int64), there.astype(np.float64)[:, None], np.zeros(len(target)), there


def mean_weights(there):
    n = int(there.sum())
    return there / max(1, n)


SHAPES = [
    (1, 64, 1),            # one row, one id: p = 1
    (1, 8, 7),             # the smallest product
    (3, 72, 64),           # a whole piece
    (130, 72, 65),         # one row tile and two rows, one column more than a piece
    (256, 64, 512),        # the tiny model's batch
    (300, 520, 1003),      # ragged in every dimension, split products
    (512, 256, 4096),      # several tiles of an SM pair
    (1000, 136, 2501),     # the same, ragged
    (17, 2048, 700),       # few rows, long sums
]


@gpu
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("T,d,V", SHAPES)
def test_cross_entropy_against_its_definition(T, d, V, weights):
    import torch
    from paper_2509_22418_b200 import ppu
    rng, Xt, X, Et, E, target = make(T, d, V, seed=T + 3 * d + 7 * V)
    if T > 2:
        target[rng.random(T) < 0.25] = -1
        target[1] = -100
    ids, q, ent, there = hard(target)
    w = (rng.random(T) + 0.5).astype(np.float32) / np.float32(T) if weights else None
    w64 = w.astype(np.float64) * there if weights else mean_weights(there)
    R = definition(X, E, ids, q, ent, w64, 1.0)
    tol = tolerances(X, E, q, w64, 1.0, R, ent)
    R["row"] = R["row"] * there
    tol["row"] = tol["row"] * there       # rows that do not count: exactly 0
    wt = torch.from_numpy(w).cuda() if weights else None
    tt = torch.from_numpy(target).cuda()
    check(ppu.ppu_head_xent(Xt, Et, tt, row_weight=wt), R, tol)
    got = ppu.ppu_head_xent(Xt, Et, tt, row_weight=wt, grad=False)
    assert got[3] is None and got[4] is None
    check(got, R, tol)


@gpu
@pytest.mark.parametrize("which", ["x", "e"])
def test_one_gradient_alone_has_the_same_bits(which):
    import torch
    from paper_2509_22418_b200 import ppu
    _, Xt, _, Et, _, target = make(300, 64, 1003, seed=4)
    tt = torch.from_numpy(target).cuda()
    both = ppu.ppu_head_xent(Xt, Et, tt)
    one = ppu.ppu_head_xent(Xt, Et, tt, grad=which)
    i = 3 if which == "x" else 4
    assert torch.equal(one[i], both[i]) and one[7 - i] is None
    for j in range(3):
        assert torch.equal(one[j], both[j])


@gpu
@pytest.mark.parametrize("T,d,V", [(1000, 64, 1003), (769, 264, 2500), (513, 256, 4096)])
def test_chunks_of_rows(T, d, V):
    """Several chunks: the vocabulary matrix's gradient is a running sum over them."""
    import torch
    from paper_2509_22418_b200 import ppu
    rng, Xt, X, Et, E, target = make(T, d, V, seed=T)
    target[rng.random(T) < 0.2] = -1
    target[256:512] = -1                   # a whole chunk without a target
    ids, q, ent, there = hard(target)
    w = mean_weights(there)
    R = definition(X, E, ids, q, ent, w, 1.0)
    tol = tolerances(X, E, q, w, 1.0, R, ent)
    R["row"] *= there
    tol["row"] *= there
    tt = torch.from_numpy(target).cuda()
    whole = ppu.ppu_head_xent(Xt, Et, tt)
    for rows in (1, 256, 300, 1 << 20):
        got = ppu.ppu_head_xent(Xt, Et, tt, chunk_rows=rows)
        check(got, R, tol)
        for j in range(3):
            assert torch.equal(got[j], whole[j])


@gpu
@pytest.mark.parametrize("T,d,V", [
    (1001, 72, 5003),      # a last wave of a few tiles, worked as halves
    (1100, 40, 9001),      # the same behind more than two tiles a block
    (100, 64, 40001),      # one row tile, wide tiles
    (100, 200, 80003),     # the same, three tiles a block
    (700, 136, 33000),     # five tiles a block
])
def test_how_tiles_are_shared_out(T, d, V):
    import torch
    from paper_2509_22418_b200 import ppu
    rng, Xt, X, Et, E, target = make(T, d, V, seed=T + d)
    target[2::5] = -1
    ids, q, ent, there = hard(target)
    w = mean_weights(there)
    R = definition(X, E, ids, q, ent, w, 1.0)
    tol = tolerances(X, E, q, w, 1.0, R, ent)
    R["row"] *= there
    tol["row"] *= there
    check(ppu.ppu_head_xent(Xt, Et, torch.from_numpy(target).cuda()), R, tol)


@gpu
def test_large_vocabulary():
    import torch
    from paper_2509_22418_b200 import ppu
    T, d, V = 600, 64, 140003
    rng, Xt, X, Et, E, target = make(T, d, V, seed=9)
    target[5::7] = -1
    ids, q, ent, there = hard(target)
    w = mean_weights(there)
    R = definition(X, E, ids, q, ent, w, 1.0)
    tol = tolerances(X, E, q, w, 1.0, R, ent)
    R["row"] *= there
    tol["row"] *= there
    check(ppu.ppu_head_xent(Xt, Et, torch.from_numpy(target).cuda()), R, tol)


@gpu
def test_offsets_beyond_32_bits():
    """A chunk of more than 2^31 kept values, and the same in small chunks.  (Beside bf16 steps of the
    results the two forms' dE differ by their fp32 sums' order, up to (T / 16 + 12) 2^-23 of the sum of
    magnitudes, which exceeds a step where the sum cancels; so each is held to the definition.)"""
    import torch
    from paper_2509_22418_b200 import ppu
    T, d, V = 16512, 64, 132000
    g = torch.Generator(device="cuda").manual_seed(3)
    E = (torch.randn((V, d), generator=g, device="cuda") * (3.0 / 8)).bfloat16()
    target = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    X = (torch.randn((T, d), generator=g, device="cuda") + 0.8 * E[target.long()].float()).bfloat16()
    got = ppu.ppu_head_xent(X, E, target, chunk_rows=T)
    small = ppu.ppu_head_xent(X, E, target, chunk_rows=512)
    assert torch.equal(got[1], small[1]) and torch.equal(got[2], small[2])
    # definition and tolerances as above, by blocks of rows on the device
    x, e = X.double(), E.double()
    R = {n: torch.zeros(*z, dtype=torch.float64, device="cuda") for n, z in (("row", (T,)), ("lse", (T,)), ("dX", (T, d)), ("dE", (V, d)))}
    tol = {n: torch.zeros_like(z) for n, z in R.items()}
    w, sums = 1.0 / T, lambda n: (n / 16 + 12) * 2 * U
    for a in range(0, T, 512):
        b = slice(a, min(T, a + 512))
        s = x[b] @ e.T
        s_err = (d / 16 + 8) * 2 * U * (x[b].abs() @ e.abs().T) + 2 * U * s.abs()
        lse = torch.logsumexp(s, 1)
        at = (torch.arange(len(s), device="cuda"), target[b].long())
        spread, worst = s.abs().amax(1) + lse.abs(), s_err.amax(1)
        R["lse"][b], R["row"][b] = lse, lse - s[at]
        tol["lse"][b] = worst + 2.0 ** -21 + 4 * U * spread + 8 * U
        tol["row"][b] = tol["lse"][b] + worst + 32 * U * (spread + 8)
        p = torch.exp(s - lse[:, None])
        ds = p * w
        ds[at] -= w
        err = w * p * (2 * BF + 2.0 ** -14 + 1.01 * (s_err + tol["lse"][b][:, None])) + BF * ds.abs() + w * 64 * U
        R["dX"][b] = ds @ e
        tol["dX"][b] = (err @ e.abs() + sums(V) * (ds.abs() @ e.abs())) * (1 + BF) + BF * R["dX"][b].abs()
        R["dE"] += ds.T @ x[b]
        err = err * (1 + BF) + BF * ds.abs()
        tol["dE"] += (err.T @ x[b].abs() + sums(T) * (ds.abs().T @ x[b].abs())) * (1 + BF)
    tol["dE"] += BF * R["dE"].abs()
    for out in (got, small):
        for n, o in zip(("row", "lse", "dX", "dE"), out[1:]):
            bad = (o.double() - R[n]).abs() > tol[n] + 1e-30
            assert not bool(bad.any()), (n, int(bad.sum()))


def teacher(rng, T, V, k, target, ragged):
    ids = rng.integers(0, V, (T, k)).astype(np.int32)
    ids[:, 0] = target
    if k > 2:
        ids[:, 2] = ids[:, 1]              # an id given twice
    z = (rng.standard_normal((T, k)) * 1.5 + 6.0).astype(np.float32)
    if ragged:
        for t in range(T):
            n = rng.integers(0, k + 1)
            ids[t, n:] = -1
            z[t, n:] = [np.nan, np.inf, -np.inf, 1e30][t % 4]     # what stands in absent places is not read
        z[::5, 0] = -np.inf                # an entry that is there by its id alone
    return ids, z


def soft(ids, z, temp, lse):
    z = z.astype(np.float64) / temp
    there = (ids >= 0) & ~(z == -np.inf)
    zz = np.where(there, z, -np.inf)
    if lse is None:
        m = np.where(there.any(1), zz.max(1, initial=-np.inf), 0.0)[:, None]
        norm = m + np.log(np.maximum(np.exp(zz - m).sum(1, keepdims=True), 1e-300))
    else:
        norm = lse.astype(np.float64)[:, None]
    logq = np.where(there, zz - norm, 0.0)
    q = np.where(there, np.exp(logq), 0.0)
    return np.maximum(ids, 0).astype(np.int64), q, (q * logq).sum(1), there.any(1)


@gpu
@pytest.mark.parametrize("T,d,V,k,temp,ragged,known", [
    (1, 64, 130, 1, 1.0, False, False),
    (5, 8, 7, 6, 2.0, True, False),
    (130, 72, 65, 5, 1.5, True, True),
    (300, 520, 1003, 32, 4.0, True, False),
    (512, 256, 4096, 64, 2.0, False, True),
    (257, 128, 600, 128, 0.7, True, False),
])
def test_distillation_against_its_definition(T, d, V, k, temp, ragged, known):
    import torch
    from paper_2509_22418_b200 import ppu
    rng, Xt, X, Et, E, target = make(T, d, V, seed=T + k)
    ids, z = teacher(rng, T, V, k, target, ragged)
    lse = (np.log(np.exp(np.where((ids >= 0) & np.isfinite(z), z, -50.0).astype(np.float64) / temp).sum(1)) + 0.1 + rng.random(T)).astype(np.float32) if known else None
    ii, q, ent, there = soft(ids, z, temp, lse)
    for weights in (False, True):
        w = rng.random(T).astype(np.float32) if weights else None
        w64 = w.astype(np.float64) * there if weights else mean_weights(there)
        R = definition(X, E, ii, q, ent, w64, temp)
        tol = tolerances(X, E, q, w64, temp, R, ent)
        # the teacher's side: q from fp32 exponentials of scaled logits, (|z| / temp + |norm| + 8) roundings
        rel = 16 * U * (8 + np.abs(np.where(q > 0, z, 0.0)).max(1) / temp + (np.abs(lse) if known else 8.0) + np.log(k + 1))
        tol["row"] = (tol["row"] + rel * (np.abs(ent) + R["Q"] * (np.abs(R["lse"]) + np.abs(R["s"]).max(1) + 4))) * there
        tol["loss"] += (np.abs(w64) * tol["row"]).sum()
        tol["dX"] += (np.abs(w64) * rel * R["Q"])[:, None] * 2 * np.abs(E).max(0)[None] / temp
        extra = np.zeros_like(R["ds"])
        np.add.at(extra, (np.arange(T)[:, None], ii), q)
        tol["dE"] += ((extra + R["Q"][:, None] * R["p"]) * (np.abs(w64) * rel)[:, None]).T @ np.abs(X) / temp
        R["row"] = R["row"] * there
        got = ppu.ppu_head_distill(Xt, Et, torch.from_numpy(ids).cuda(), torch.from_numpy(z).cuda(), temperature=temp,
                                   teacher_lse=None if lse is None else torch.from_numpy(lse).cuda(),
                                   row_weight=None if w is None else torch.from_numpy(w).cuda())
        check(got, R, tol)


@gpu
@pytest.mark.parametrize("T,d,V,k", [(700, 72, 1003, 5), (1024, 8, 64, 128), (600, 64, 300, 2), (1300, 40, 500, 3)])
@pytest.mark.parametrize("weights", [False, True])
def test_distillation_in_chunks_of_rows(T, d, V, k, weights):
    """A mean counts the rows of all chunks: loss and row factors as with one chunk."""
    import torch
    from paper_2509_22418_b200 import ppu
    rng, Xt, X, Et, E, target = make(T, d, V, seed=T)
    ids, z = teacher(rng, T, V, k, target, True)
    ids[256:512] = -1                      # a whole chunk without an entry
    ii, q, ent, there = soft(ids, z, 1.0, None)
    w = rng.random(T).astype(np.float32) if weights else None
    w64 = w.astype(np.float64) * there if weights else mean_weights(there)
    R = definition(X, E, ii, q, ent, w64, 1.0)
    args = [Xt, Et, torch.from_numpy(ids).cuda(), torch.from_numpy(z).cuda()]
    wt = None if w is None else torch.from_numpy(w).cuda()
    whole = ppu.ppu_head_distill(*args, row_weight=wt)
    assert abs(float(whole[0]) - (w64 * R["row"]).sum()) <= 1e-3 * (np.abs(w64) * np.abs(R["row"])).sum()
    # dE: fp32 sums of the same products in another order, 2^-23 a term and side, each rounded once to bf16
    tol = 2 * BF * whole[4].double().abs().cpu().numpy() * (1 + 2 * BF) + 2 * T * 2 * U * (np.abs(R["ds"]).T @ np.abs(X)) * (1 + 8 * BF)
    for rows in (1, 512):
        got = ppu.ppu_head_distill(*args, row_weight=wt, chunk_rows=rows)
        for j in range(4):
            assert torch.equal(got[j], whole[j]), j
        assert ((got[4].double() - whole[4].double()).abs().cpu().numpy() <= tol + 1e-30).all()


@gpu
def test_one_teacher_entry_is_cross_entropy():
    import torch
    from paper_2509_22418_b200 import ppu
    _, Xt, _, Et, _, target = make(300, 72, 1003, seed=2)
    target[::3] = -1
    tt = torch.from_numpy(target).cuda()
    a = ppu.ppu_head_xent(Xt, Et, tt)
    b = ppu.ppu_head_distill(Xt, Et, tt[:, None], torch.full((300, 1), 3.5, device="cuda"))
    for x, y in zip(a, b):
        assert torch.equal(x, y)


@gpu
def test_no_row_counts():
    import torch
    from paper_2509_22418_b200 import ppu
    _, Xt, X, Et, E, _ = make(70, 64, 200, seed=1)
    none = torch.full((70,), -1, dtype=torch.int32, device="cuda")
    nan = torch.full((70,), float("nan"), device="cuda")      # the weight of a row that does not count is not used
    for w in (None, nan):
        loss, row, lse, dX, dE = ppu.ppu_head_xent(Xt, Et, none, row_weight=w)
        assert float(loss) == 0 and not row.any() and not dX.any() and not dE.any()
        s = X @ E.T
        assert np.allclose(lse.cpu().numpy(), np.log(np.exp(s).sum(1)), rtol=1e-5)
    loss, row, lse, dX, dE = ppu.ppu_head_distill(Xt, Et, none[:, None], nan[:, None])
    assert float(loss) == 0 and not row.any() and not dX.any() and not dE.any()
    # no rows at all
    loss, row, lse, dX, dE = ppu.ppu_head_xent(Xt[:0], Et, none[:0])
    assert float(loss) == 0 and row.shape == (0,) and dX.shape == (0, 64) and not dE.any()


@gpu
def test_ids_outside_the_vocabulary_are_left_out_and_reported():
    import torch
    from paper_2509_22418_b200 import ppu
    _, Xt, _, Et, _, target = make(70, 64, 200, seed=6)
    flags = torch.zeros(8, dtype=torch.int32, device="cuda")
    good = torch.from_numpy(target).cuda()
    ppu.ppu_head_xent(Xt, Et, good, flags=flags)
    ppu.ppu_op_status(flags)
    bad, left_out = good.clone(), good.clone()
    bad[3], bad[69], left_out[3], left_out[69] = 200, 2 ** 31 - 1, -1, -1
    got = ppu.ppu_head_xent(Xt, Et, bad, flags=flags)
    with pytest.raises(ppu.PpuError) as e:
        ppu.ppu_op_status(flags)
    assert e.value.code == -8
    ppu.ppu_op_status(flags)               # cleared
    for a, b in zip(got, ppu.ppu_head_xent(Xt, Et, left_out)):
        assert torch.equal(a, b)
    ids = torch.stack([good, bad], 1)
    z = torch.ones((70, 2), device="cuda")
    got = ppu.ppu_head_distill(Xt, Et, ids, z, flags=flags)
    with pytest.raises(ppu.PpuError):
        ppu.ppu_op_status(flags)
    for a, b in zip(got, ppu.ppu_head_distill(Xt, Et, torch.stack([good, left_out], 1), z)):
        assert torch.equal(a, b)


@gpu
def test_confident_and_hopeless_rows():
    """Rows where the target has all of the probability, and rows hundreds of nats away from it: beyond the
    range of the powers' common reference."""
    import torch
    from paper_2509_22418_b200 import ppu
    T, d, V = 64, 64, 300
    rng = np.random.default_rng(8)
    Et, E = bf16(np.sign(rng.standard_normal((V, d))))
    target = rng.integers(0, V, T).astype(np.int32)
    Xt, X = bf16(E[target] * np.where(np.arange(T) % 2 == 0, 4.0, -4.0)[:, None])    # target logit +-256, others within about +-160
    ids, q, ent, there = hard(target)
    w = mean_weights(there)
    R = definition(X, E, ids, q, ent, w, 1.0)
    assert R["row"].max() > 300 and R["row"].min() < 1e-6
    check(ppu.ppu_head_xent(Xt.cuda(), Et.cuda(), torch.from_numpy(target).cuda()), R, tolerances(X, E, q, w, 1.0, R, ent))


@gpu
@pytest.mark.parametrize("shift", [-90.0, -45.0, 45.0, 90.0])
def test_logits_far_from_zero(shift):
    """Rows whose logits all lie far from zero, rows with some pieces there, and ordinary rows together."""
    import torch
    from paper_2509_22418_b200 import ppu
    T, d, V = 200, 72, 1003
    rng = np.random.default_rng(int(shift) + 100)
    E = rng.standard_normal((V, d)) * (3.0 / math.sqrt(d))
    E[:, 0] = 1.0                          # a row's first value is added to all of its logits
    E[:, 1] = np.where(np.arange(V) // 64 % 3 == 1, 1.0, 0.0)      # the second to every third piece's
    Et, E = bf16(E)
    x = rng.standard_normal((T, d))
    x[:, 0] = np.where(np.arange(T) % 2 == 0, shift, 0.0)
    x[:, 1] = np.where(np.arange(T) % 3 == 0, -shift, 0.0)
    Xt, X = bf16(x)
    target = rng.integers(0, V, T).astype(np.int32)
    target[5::9] = -1
    ids, q, ent, there = hard(target)
    w = mean_weights(there)
    R = definition(X, E, ids, q, ent, w, 1.0)
    tol = tolerances(X, E, q, w, 1.0, R, ent)
    R["row"] *= there
    tol["row"] *= there
    check(ppu.ppu_head_xent(Xt.cuda(), Et.cuda(), torch.from_numpy(target).cuda()), R, tol)


@gpu
@pytest.mark.parametrize("size,temp", [(30, 1.0), (200, 1.0), (1e3, 1.0), (30, 1e-3), (3e3, 1.0), (1e6, 1.0), (1e4, 1e-4), (1e12, 1.0)])
def test_logits_whose_roundings_are_large(size, temp):
    """Logits of 1e4 to 1e26: the softmax is the largest logit's, losses are differences of logits."""
    import torch
    from paper_2509_22418_b200 import ppu
    rng = np.random.default_rng(5)
    T, d, V = 260, 64, 500
    Xt, X = bf16(rng.standard_normal((T, d)) * size)
    Et, E = bf16(rng.standard_normal((V, d)) * size)
    target = rng.integers(0, V, T).astype(np.int32)
    s = X @ E.T / temp
    order = np.argsort(s, 1)
    top = order[:, -1]
    target[::4] = top[::4]
    mag = (np.abs(X) @ np.abs(E).T).max(1) / temp
    err = (d / 16 + 12) * 2 * U * mag      # of a logit, its scaling included
    r = np.arange(T)
    clear = s[r, top] - s[r, order[:, -2]] > 2 * err + 100
    assert clear.mean() > 0.9
    X, target, top, s, err, mag = X[clear], target[clear], top[clear], s[clear], err[clear], mag[clear]
    T = len(X)
    r = np.arange(T)
    tt = torch.from_numpy(target).cuda()
    Xc, Ec = torch.from_numpy(X).bfloat16().cuda(), Et.cuda()
    if temp == 1.0:
        loss, row, lse, dX, dE = ppu.ppu_head_xent(Xc, Ec, tt)
    else:
        loss, row, lse, dX, dE = ppu.ppu_head_distill(Xc, Ec, tt[:, None], torch.ones(T, 1, device="cuda"), temperature=temp)
    assert (np.abs(lse.double().cpu().numpy() - s[r, top]) <= err + 4).all()
    assert (np.abs(row.double().cpu().numpy() - (s[r, top] - s[r, target])) <= 2 * err + 8).all()
    # the target's own power, 2^y with |y| <= 1/2 (its distance from the rounded reference), is off by 2^-22, and so is
    # y - log2 of it, with the roundings of y and of the logarithm (2^-25 each): below 2^-21, and nothing else adds to it
    assert (np.abs(row.cpu().numpy()[target == top]) <= 2.0 ** -20).all()
    # two powers, one factor and the result are rounded to bf16
    want, size_of = (E[top] - E[target]) / T / temp, (np.abs(E[top]) + np.abs(E[target])) / T / temp
    assert (np.abs(dX.double().cpu().numpy() - want) <= 4 * BF * size_of).all()
    ds = np.zeros((T, V))
    ds[r, top] += 1 / T / temp
    np.add.at(ds, (r, target), -1 / T / temp)
    one = np.zeros((T, V))
    one[r, top] = one[r, target] = 1 / T / temp
    one[target == top] *= 2.0 ** -20 / (5 * BF)            # (there p - 1, off as the loss is)
    assert (np.abs(dE.double().cpu().numpy() - ds.T @ X) <= 5 * BF * (one.T @ np.abs(X))).all()


@gpu
def test_rows_that_do_not_count_may_hold_anything():
    import torch
    from paper_2509_22418_b200 import ppu
    _, Xt, _, Et, _, target = make(300, 72, 1003, seed=14)
    target[::4] = -1
    tt = torch.from_numpy(target).cuda()
    Xz = Xt.clone()
    Xz[::4] = 0
    ref = ppu.ppu_head_xent(Xz, Et, tt)
    for junk in (float("nan"), float("inf"), 3e38):
        Xj = Xt.clone()
        Xj[::4] = junk
        for chunk in (0, 256):
            got = ppu.ppu_head_xent(Xj, Et, tt, chunk_rows=chunk)
            ref = ppu.ppu_head_xent(Xz, Et, tt, chunk_rows=chunk)
            for i in (0, 1, 3, 4):
                assert torch.equal(got[i], ref[i]), (junk, i)


@gpu
def test_gradients_against_differences():
    """The loss itself at steps that bf16 holds exactly (values are multiples of 1/8, steps of 1/8)."""
    import torch
    from paper_2509_22418_b200 import ppu
    T, d, V = 96, 64, 333
    rng = np.random.default_rng(12)
    grid = lambda *s: np.clip(np.round(rng.standard_normal(s) * 8), -16, 16) / 8  # noqa: E731
    X, E = grid(T, d), grid(V, d) / 4
    target = torch.from_numpy(rng.integers(0, V, T).astype(np.int32)).cuda()
    ids = torch.from_numpy(rng.integers(0, V, (T, 5)).astype(np.int32)).cuda()
    z = torch.from_numpy(rng.standard_normal((T, 5)).astype(np.float32)).cuda()
    ones = torch.full((T,), 1.0 / T, device="cuda")

    def loss(call, x, e):
        return call(bf16(x)[0].cuda(), bf16(e)[0].cuda())
    calls = [lambda x, e: ppu.ppu_head_xent(x, e, target), lambda x, e: ppu.ppu_head_distill(x, e, ids, z, temperature=2.0, row_weight=ones)]
    for call in calls:
        got = loss(call, X, E)
        for i, (at, step) in enumerate(((X, 1 / 8), (E, 1 / 32))):
            grad = got[3 + i].double().cpu().numpy()
            for trial in range(4):
                D = np.zeros_like(at)
                rows = rng.integers(0, len(at), 6)
                if i == 1:                 # rows of E that carry a gradient: targets and teacher entries
                    rows = (target if trial % 2 else ids[:, 0]).cpu().numpy()[rng.integers(0, T, 6)]
                D[rows, rng.integers(0, d, 6)] = step
                plus, minus = ((X + D, E), (X - D, E)) if i == 0 else ((X, E + D), (X, E - D))
                diff = float(loss(call, *plus)[0].double() - loss(call, *minus)[0].double()) / 2
                want = float((grad * D).sum())
                # third derivatives of a log-sum-exp are at most 1 / 4 of the step cubed (times the logit's change, at most
                # 2 * 6 steps), fp32 losses about 6 give 4e-7 each, the gradient's elements 2 * 2^-8 and more
                size = float((np.abs(grad) * np.abs(D)).sum())
                bound = 4 * BF * size + 2e-6 + (12 * step) ** 3 / 24 / T
                assert abs(diff - want) <= bound, (i, trial, diff, want, bound)


@gpu
def test_strided_operands_and_untouched_surroundings():
    """Row strides on every operand; the padding of dX and dE and the bytes behind them keep their values."""
    import torch
    from paper_2509_22418_b200 import ppu
    T, d, V, k = 300, 72, 1003, 7
    rng, Xt, X, Et, E, target = make(T, d, V, seed=21)
    ids, z = teacher(rng, T, V, k, target, True)
    idt, zt = torch.from_numpy(ids).cuda(), torch.from_numpy(z).cuda()
    ref = ppu.ppu_head_distill(Xt, Et, idt, zt, temperature=1.5)
    wide = lambda t, n: torch.cat([t, torch.full((t.shape[0], n), 77, dtype=t.dtype, device="cuda")], 1)[:, : t.shape[1]]  # noqa: E731
    Xs, Es, ids_s, zs = wide(Xt, 24), wide(Et, 8), wide(idt, 3), wide(zt, 5)
    got = ppu.ppu_head_distill(Xs, Es, ids_s, zs, temperature=1.5)
    for a, b in zip(ref, got):
        assert torch.equal(a, b)
    # the C call with strided outputs
    dX = torch.full((T + 1, d + 16), 5.0, dtype=torch.bfloat16, device="cuda")
    dE = torch.full((V + 1, d + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    nb = ppu.ppu_head_query_bytes(T, d, V, k=k)
    ws = torch.full((nb + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    out = torch.full((2 * T + 1 + 8,), 9.0, device="cuda")
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    i64 = C.c_int64
    rc = ppu.lib().ppu_head_distill(p(Xs), i64(Xs.stride(0)), p(Es), i64(Es.stride(0)), p(ids_s), i64(ids_s.stride(0)), p(zs), i64(zs.stride(0)), k,
                                    None, C.c_float(1.5), None, T, d, V, p(out), p(out[1:]), p(out[1 + T:]), p(dX), i64(d + 16), p(dE), i64(d + 8), 0,
                                    p(ws), C.c_size_t(nb), None, C.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert rc == 0
    torch.cuda.synchronize()
    assert torch.equal(dX[:T, :d], ref[3]) and torch.equal(dE[:V, :d], ref[4])
    assert bool((dX[:, d:] == 5).all()) and bool((dX[T] == 5).all()) and bool((dE[:, d:] == 5).all()) and bool((dE[V] == 5).all())
    assert float(out[0]) == float(ref[0]) and torch.equal(out[1:1 + T], ref[1]) and torch.equal(out[1 + T:1 + 2 * T], ref[2])
    assert bool((out[1 + 2 * T:] == 9).all()) and bool((ws[nb:] == 0xA5).all())


@gpu
@pytest.mark.parametrize("T,chunk", [(20000, 0), (1500, 256), (0, 0)])
def test_capture_of_counted_rows_and_chunks(T, chunk):
    """Rows counted by a kernel of their own (behind a memset for many), several chunks, no rows at all."""
    import torch
    from paper_2509_22418_b200 import ppu
    g = torch.Generator(device="cuda").manual_seed(3)
    X = torch.randn(T, 64, generator=g, device="cuda").bfloat16()
    E = (torch.randn(300, 64, generator=g, device="cuda") * 0.4).bfloat16()
    ids = torch.randint(-50, 300, (T, 3), generator=g, device="cuda", dtype=torch.int32)
    z = torch.randn(T, 3, generator=g, device="cuda")
    calls = [lambda: ppu.ppu_head_xent(X, E, ids[:, 0].contiguous(), chunk_rows=chunk), lambda: ppu.ppu_head_distill(X, E, ids, z, chunk_rows=chunk)]
    for call in calls:
        want = [t.clone() for t in call()]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            call()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                got = call()
            for t in got:
                t.fill_(7)
            for _ in range(2):
                graph.replay()
        s.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@gpu
def test_captured_streamed_and_repeated_calls_have_the_same_bits():
    import torch
    from paper_2509_22418_b200 import ppu
    _, Xa, _, Ea, _, ta = make(300, 136, 2501, seed=31)
    _, Xb, _, Eb, _, tb = make(300, 136, 2501, seed=32)
    ta, tb = torch.from_numpy(ta).cuda(), torch.from_numpy(tb).cuda()
    ref_a, ref_b = ppu.ppu_head_xent(Xa, Ea, ta), ppu.ppu_head_xent(Xb, Eb, tb)
    again = ppu.ppu_head_xent(Xa, Ea, ta)
    assert all(torch.equal(x, y) for x, y in zip(ref_a, again))
    # two calls at once on two streams
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    s1.wait_stream(torch.cuda.current_stream())
    s2.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(s1):
            got_a = ppu.ppu_head_xent(Xa, Ea, ta)
        with torch.cuda.stream(s2):
            got_b = ppu.ppu_head_xent(Xb, Eb, tb)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(ref_a, got_a))
    assert all(torch.equal(x, y) for x, y in zip(ref_b, got_b))
    # captured once, replayed on new values
    X, E, t = Xa.clone(), Ea.clone(), ta.clone()
    ws = torch.empty(ppu.ppu_head_query_bytes(300, 136, 2501), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ppu.ppu_head_xent(X, E, t, workspace=ws)
    for x, e, tt, ref in ((Xb, Eb, tb, ref_b), (Xa, Ea, ta, ref_a), (Xb, Eb, tb, ref_b)):
        X.copy_(x), E.copy_(e), t.copy_(tt)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref))


# ---- refusals, on the host ----------------------------------------------------------------------
@pytest.fixture(scope="module")
def ppu():
    from paper_2509_22418_b200 import build, ppu as mod
    build.build()
    return mod


def test_sizes_of_the_workspace(ppu):
    q = ppu.ppu_head_query_bytes
    full = 8192 * 32768 * 2
    assert q(8192, 2048, 32768, 0) < full / 15           # statistics of the pieces (8 bytes for 64 values) and the rows
    assert q(8192, 2048, 32768, 1) < 0.75 * full         # half of the rows' softmax beside them
    # a chunk's softmax (6144 rows), dE's running sum and fX, and a few values for each row, however many rows
    assert q(1 << 20, 2048, 32768, 3) < 6144 * (32768 * 2 + 512 * 8 + 2048 * 2) + 32768 * 2048 * 4 + 16 * (1 << 20)
    assert q(1 << 20, 8, 1 << 22, 1) < 1.2 * 2 ** 31
    assert q(8192, 2048, 32768, 3, chunk_rows=256) < q(8192, 2048, 32768, 3)
    for bad in [(1, 12, 8), (1, 0, 8), (1, 16392, 8), (-1, 8, 8), (1, 8, 0), ((1 << 20) + 1, 8, 8), (1, 8, (1 << 22) + 1)]:
        with pytest.raises(ppu.PpuError):
            q(*bad)
    for kw in (dict(grads=4), dict(grads=-1), dict(chunk_rows=-1), dict(k=0), dict(k=129)):
        with pytest.raises(ppu.PpuError):
            q(8, 8, 8, **kw)


def _xent(ppu, **change):
    """A call on host addresses that must be refused before anything is launched."""
    buf = (C.c_uint8 * 65536)()
    base = (C.addressof(buf) + 255) & ~255
    a = dict(X=base, ldx=64, E=base, lde=64, target=base, w=None, T=4, d=64, V=32, loss=base, row=base, lse=base, dX=base, lddx=64, dE=base, ldde=64,
             chunk=0, ws=base, nb=1 << 40, flags=None)
    a.update(change)
    v, i64 = C.c_void_p, C.c_int64
    return ppu.lib().ppu_head_xent(v(a["X"]), i64(a["ldx"]), v(a["E"]), i64(a["lde"]), v(a["target"]), v(a["w"]), a["T"], a["d"], a["V"], v(a["loss"]),
                                   v(a["row"]), v(a["lse"]), v(a["dX"]), i64(a["lddx"]), v(a["dE"]), i64(a["ldde"]), a["chunk"], v(a["ws"]),
                                   C.c_size_t(a["nb"]), v(a["flags"]), None)


@pytest.mark.parametrize("change,code", [
    (dict(X=None), -1), (dict(E=None), -1), (dict(target=None), -1), (dict(loss=None), -1), (dict(ws=None), -1),
    (dict(ldx=56), -1), (dict(ldx=68), -1), (dict(lde=60), -1), (dict(lddx=8), -1), (dict(ldde=65), -1),
    (dict(d=60), -2), (dict(d=0), -1), (dict(V=0), -1), (dict(T=-1), -1), (dict(chunk=-5), -1), (dict(nb=64), -4),
])
def test_cross_entropy_refuses(ppu, change, code):
    assert _xent(ppu, **change) == code and ppu.lib().ppu_last_error()


def test_cross_entropy_refuses_misaligned_operands(ppu):
    buf = (C.c_uint8 * 65536)()
    base = (C.addressof(buf) + 255) & ~255
    for name in ("X", "E", "dX", "dE"):
        assert _xent(ppu, **{name: base + 8}) == -1
    assert _xent(ppu, ws=base + 16) == -1


@pytest.mark.parametrize("k,ldi,ldz,temp,z,code", [(0, 4, 4, 1.0, True, -2), (129, 200, 200, 1.0, True, -2), (4, 3, 4, 1.0, True, -1), (4, 4, 3, 1.0, True, -1),
                                                   (4, 4, 4, 0.0, True, -1), (4, 4, 4, -1.0, True, -1), (4, 4, 4, math.nan, True, -1),
                                                   (4, 4, 4, math.inf, True, -1), (4, 4, 4, 1e-5, True, -1), (4, 4, 4, 1e5, True, -1),
                                                   (4, 4, 4, 1.0, False, -1)])
def test_distillation_refuses(ppu, k, ldi, ldz, temp, z, code):
    buf = (C.c_uint8 * 4096)()
    base = (C.addressof(buf) + 255) & ~255
    v, i64 = C.c_void_p, C.c_int64
    rc = ppu.lib().ppu_head_distill(v(base), i64(64), v(base), i64(64), v(base), i64(ldi), v(base if z else None), i64(ldz), k, None, C.c_float(temp), None,
                                    4, 64, 32, v(base), None, None, None, i64(64), None, i64(64), 0, v(base), C.c_size_t(1 << 30), None, None)
    assert rc == code


def test_tensors_are_checked(ppu):
    import torch
    X, E, t = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(32, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: ppu.ppu_head_xent(X, E, t), lambda: ppu.ppu_head_distill(X, E, t[:, None], X[:, :1].float()), lambda: ppu.ppu_op_status(t)):
        with pytest.raises(ppu.PpuError):
            call()


@gpu
def test_device_tensors_are_checked():
    import torch
    from paper_2509_22418_b200 import ppu
    z = lambda *s, **k: torch.zeros(s, device="cuda", **k)  # noqa: E731
    b = torch.bfloat16
    X, E, t = z(4, 64, dtype=b), z(32, 64, dtype=b), z(4, dtype=torch.int32)
    bad = [
        (X.float(), E, t), (X, E.float(), t), (X, E, t.long()), (X, E, t[:3]), (X, E[:, :56], t), (X, E.cpu(), t), (X, E, t.cpu()),
        (X.t(), E, t), (X[0], E, t), (z(64, 4, dtype=b).t(), E, t), (X, E, z(8, dtype=torch.int32)[::2]), (z(4, 60, dtype=b), z(32, 60, dtype=b), t),
        (z(4, 72, dtype=b)[:, 4:68], E, t), (z(4, 68, dtype=b)[:, :64], E, t), (z(1, 64, dtype=b).expand(4, 64), E, t),
    ]
    for args in bad:
        with pytest.raises(ppu.PpuError):
            ppu.ppu_head_xent(*args)
    for kw in (dict(row_weight=z(3)), dict(row_weight=z(4, dtype=b)), dict(flags=z(8)), dict(flags=z(4, dtype=torch.int32)),
               dict(workspace=z(16, dtype=torch.uint8)), dict(workspace=z(1 << 20)), dict(chunk_rows=-1)):
        with pytest.raises(ppu.PpuError):
            ppu.ppu_head_xent(X, E, t, **kw)
    ids, zt = z(4, 3, dtype=torch.int32), z(4, 3)
    for args in ((X, E, ids, zt[:, :2]), (X, E, ids.long(), zt), (X, E, ids, zt.double()), (X, E, t, zt), (X, E, z(4, 129, dtype=torch.int32), z(4, 129))):
        with pytest.raises(ppu.PpuError):
            ppu.ppu_head_distill(*args)
    for kw in (dict(temperature=0.0), dict(teacher_lse=z(3)), dict(teacher_lse=z(4, dtype=b))):
        with pytest.raises(ppu.PpuError):
            ppu.ppu_head_distill(X, E, ids, zt, **kw)
