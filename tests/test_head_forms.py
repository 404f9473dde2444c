"""Forms and ranges of the head losses beside those of test_head_loss.py, by the same definition in 64 bits
and the same count of roundings."""
import threading

import numpy as np
import pytest

from test_head_loss import U, bf16, check, definition, hard, make, mean_weights, soft, teacher, tolerances

gpu = pytest.mark.gpu


def cross_entropy(X, E, target, w=None):
    """Definition and tolerances; rows without a target have no loss."""
    ids, q, ent, there = hard(target)
    w = mean_weights(there) if w is None else w * there
    R = definition(X, E, ids, q, ent, w, 1.0)
    tol = tolerances(X, E, q, w, 1.0, R, ent)
    R["row"], tol["row"] = R["row"] * there, tol["row"] * there
    return R, tol


def distillation(X, E, ids, z, temp):
    """The same for a mean over rows with entries; the teacher's q in fp32 is counted as in test_head_loss.py."""
    ii, q, ent, there = soft(ids, z, temp, None)
    w = mean_weights(there)
    R = definition(X, E, ii, q, ent, w, temp)
    tol = tolerances(X, E, q, w, temp, R, ent)
    rel = 16 * U * (16 + np.abs(np.where(q > 0, z, 0.0)).max(1) / temp + np.log(ids.shape[1] + 1))
    tol["row"] = (tol["row"] + rel * (np.abs(ent) + R["Q"] * (np.abs(R["lse"]) + np.abs(R["s"]).max(1) + 4))) * there
    tol["loss"] += (np.abs(w) * tol["row"]).sum()
    tol["dX"] += (np.abs(w) * rel * R["Q"])[:, None] * 2 * np.abs(E).max(0)[None] / temp
    extra = R["Q"][:, None] * R["p"]
    np.add.at(extra, (np.arange(len(X))[:, None], ii), q)
    tol["dE"] += (extra * (np.abs(w) * rel)[:, None]).T @ np.abs(X) / temp
    R["row"] = R["row"] * there
    return R, tol


def on_device(*arrays):
    import torch
    return [torch.from_numpy(a).cuda() for a in arrays]


@gpu
@pytest.mark.parametrize("T,V", [(64, 2048), (24, 33000)])       # one warp to a row, several
def test_entries_of_little_weight_keep_their_digits(T, V):
    """Gradients of entries that teacher and student both give 1e-5 to 1e-10: relative to their own size.  E's columns as
    above, so that dX[t, c] is ds of one id: its place (or power), the row's factor and the result are off by half a step
    each; where p and q are not within a factor 5 / 3 of one another their difference has at most four times
    the relative errors of theirs, from logits below 16 ((128 / 16 + 8) 2^-23 16 each, and of their
    sum) and a handful of roundings of q's logit below 32: 4 (2 * 3.1e-5 + 8 * 32 * 2^-24) < 2^-11."""
    import torch
    from paper_2509_22418_b200 import ppu
    d, k = 128, 64
    rng = np.random.default_rng(V + 1)
    E = np.zeros((V, d))
    E[:, 1] = np.clip(3.0 * rng.standard_normal(V), -14, 14)
    at = rng.permutation(V)[: d - 2]
    E[at, np.arange(2, d)] = 1.0
    Et, E = bf16(E)
    x = np.zeros((T, d))
    x[:, 1] = rng.uniform(0.9, 1.1, T)
    Xt, X = bf16(x)
    ids = np.array([rng.permutation(at)[:k] for _ in range(T)]).astype(np.int32)
    z = np.clip(5.0 * rng.standard_normal((T, k)), -15, 15).astype(np.float32)
    ii, q, ent, _ = soft(ids, z, 1.0, None)
    R = definition(X, E, ii, q, ent, np.ones(T), 1.0)
    got = ppu.ppu_head_distill(Xt.cuda(), Et.cuda(), *on_device(ids, z), row_weight=torch.ones(T, device="cuda"))
    full = np.zeros((T, V))
    np.put_along_axis(full, ii, q, 1)
    p, full, ds = R["p"][:, at], full[:, at], R["ds"][:, at]
    clear = np.abs(p - full) >= 0.25 * (p + full)
    assert (clear & (full > 0) & (p + full < 1e-6)).sum() > 2 * T
    rel = np.abs(got[3].double().cpu().numpy()[:, 2:] / ds - 1)[clear]
    assert rel.max() <= 3 * 2.0 ** -8 * (1 + 2.0 ** -7) + 2.0 ** -11


# Warps to a row of the row kernel: one up to some 16 thousand ids or for thousands of rows, else 4, or 16 for few rows
# of more than 64 thousand ids.
SEVERAL_WARPS = [(24, 33000), (400, 33000), (24, 70000)]


@gpu
@pytest.mark.parametrize("k", [7, 64, 128])
@pytest.mark.parametrize("T,V", SEVERAL_WARPS)
def test_several_entries_with_several_warps_to_a_row(T, V, k):
    from paper_2509_22418_b200 import ppu
    rng, Xt, X, Et, E, target = make(T, 40, V, seed=T + k)
    ids, z = teacher(rng, T, V, k, target, True)        # ragged, ids given twice, rows without an entry
    ids[3] = -1
    ids[7, : min(k, 5)] = V - 1
    R, tol = distillation(X, E, ids, z, 1.5)
    check(ppu.ppu_head_distill(Xt, Et, *on_device(ids, z), temperature=1.5), R, tol)


def far(T, V, shift):
    """Rows whose logits all lie far from zero, rows with some pieces there, and ordinary rows together."""
    rng = np.random.default_rng(int(shift) + V)
    d = 72
    E = rng.standard_normal((V, d)) * (3.0 / np.sqrt(d))
    E[:, 0] = 1.0                          # a row's first value is added to all of its logits
    E[:, 1] = np.where(np.arange(V) // 64 % 3 == 1, 1.0, 0.0)      # the second to every third piece's
    x = rng.standard_normal((T, d))
    x[:, 0] = np.where(np.arange(T) % 2 == 0, shift, 0.0)
    x[:, 1] = np.where(np.arange(T) % 3 == 0, -shift, 0.0)
    (Xt, X), (Et, E) = bf16(x), bf16(E)
    target = rng.integers(0, V, T).astype(np.int32)
    target[5::9] = -1
    return rng, Xt.cuda(), X, Et.cuda(), E, target


@gpu
@pytest.mark.parametrize("shift", [-90.0, -45.0, 45.0, 90.0])
@pytest.mark.parametrize("T,V", [(24, 33000), (130, 33000), (24, 70000)])
def test_logits_far_from_zero_with_several_warps_to_a_row(T, V, shift):
    from paper_2509_22418_b200 import ppu
    _, Xt, X, Et, E, target = far(T, V, shift)
    check(ppu.ppu_head_xent(Xt, Et, *on_device(target)), *cross_entropy(X, E, target))


@gpu
@pytest.mark.parametrize("shift", [-90.0, 45.0, 90.0])
@pytest.mark.parametrize("T,V,k", [(200, 1003, 7), (24, 33000, 64), (24, 70000, 7)])
def test_several_entries_with_logits_far_from_zero(T, V, k, shift):
    from paper_2509_22418_b200 import ppu
    rng, Xt, X, Et, E, target = far(T, V, shift)
    ids, z = teacher(rng, T, V, k, np.maximum(target, 0), True)
    ids[target < 0] = -1
    check(ppu.ppu_head_distill(Xt, Et, *on_device(ids, z)), *distillation(X, E, ids, z, 1.0))


@gpu
@pytest.mark.parametrize("T,V", SEVERAL_WARPS)
def test_rows_that_do_not_count_may_hold_anything_with_several_warps_to_a_row(T, V):
    import torch
    from paper_2509_22418_b200 import ppu
    _, Xt, _, Et, _, target = make(T, 16, V, seed=14)
    target[::4] = -1
    tt, = on_device(target)
    Xt[::4] = 0
    ref = ppu.ppu_head_xent(Xt, Et, tt)
    for junk in (float("nan"), float("inf"), 3e38):
        Xj = Xt.clone()
        Xj[::4] = junk
        got = ppu.ppu_head_xent(Xj, Et, tt)
        for i in (0, 1, 3, 4):
            assert torch.equal(got[i], ref[i]), (junk, i)


@gpu
@pytest.mark.parametrize("grad", [True, "e"])
@pytest.mark.parametrize("T,d,V", [
    (4096, 64, 300),       # four slices of the rows
    (3000, 72, 1003),      # two, neither a multiple of a block
    (4096, 512, 512),      # SM pairs (single SMs where dE is all there is)
    (3000, 520, 1003),     # SM pairs, ragged
])
def test_vocabulary_gradient_in_slices_of_the_rows(T, d, V, grad):
    """Many rows and few tiles of dE: its reduction is split and joined."""
    from paper_2509_22418_b200 import ppu
    # what the workspace has beside the powers, f X and a loss's: at least two partial sums
    rows = ppu.ppu_head_query_bytes(T, d, V, grads=2) - ppu.ppu_head_query_bytes(T, d, V, grads=0)
    assert rows >= T * ((V + 63) // 64 * 64) * 2 + 2 * T * d + 2 * 4 * V * d
    rng, Xt, X, Et, E, target = make(T, d, V, seed=T + d)
    target[rng.random(T) < 0.3] = -1
    got = ppu.ppu_head_xent(Xt, Et, *on_device(target), grad=grad)
    assert (got[3] is None) == (grad == "e")
    check(got, *cross_entropy(X, E, target))


@gpu
@pytest.mark.parametrize("grad", [False, "x", "e"])
@pytest.mark.parametrize("T,d,V,k", [
    (300, 64, 1003, 5),
    (1001, 520, 5003, 7),  # dX alone: four slices on single SMs, with dE three on SM pairs
    (512, 256, 4096, 32),  # dE alone: SM pairs
    (24, 64, 33000, 64),   # few rows: dX in 31 slices
    (9, 2048, 260, 3),
])
def test_one_gradient_or_none(T, d, V, k, grad):
    """A frozen vocabulary matrix, frozen hidden states, and the loss alone, of both losses."""
    from paper_2509_22418_b200 import ppu
    rng, Xt, X, Et, E, target = make(T, d, V, seed=T + k)
    target[4::6] = -1
    got = ppu.ppu_head_xent(Xt, Et, *on_device(target), grad=grad)
    assert (got[3] is not None) == (grad == "x") and (got[4] is not None) == (grad == "e")
    check(got, *cross_entropy(X, E, target))
    ids, z = teacher(rng, T, V, k, np.maximum(target, 0), True)
    got = ppu.ppu_head_distill(Xt, Et, *on_device(ids, z), temperature=2.0, grad=grad)
    assert (got[3] is not None) == (grad == "x") and (got[4] is not None) == (grad == "e")
    check(got, *distillation(X, E, ids, z, 2.0))


@gpu
@pytest.mark.parametrize("T,d,V", [(40, 4096, 300), (300, 4104, 1003), (24, 16384, 500), (1, 16384, 64)])
def test_long_hidden_states(T, d, V):
    from paper_2509_22418_b200 import ppu
    _, Xt, X, Et, E, target = make(T, d, V, seed=d)
    target[1::5] = -1
    check(ppu.ppu_head_xent(Xt, Et, *on_device(target)), *cross_entropy(X, E, target))


@gpu
@pytest.mark.parametrize("T,V", [(260, 1003), (24, 33000)])
def test_ids_masked_by_logits_of_minus_infinity(T, V):
    """Hidden states and ids with values whose product leaves fp32: as if these ids were not there."""
    import torch
    from paper_2509_22418_b200 import ppu
    d = 72
    rng, _, X, _, E, target = make(T, d, V, seed=V)
    masked = rng.random(V) < 0.1
    masked[64:192] = True                  # whole pieces
    masked[V - 1] = True
    X[:, 0], E[:, 0] = -3e38, np.where(masked, 100.0, 0.0)
    (Xt, X), (Et, E) = bf16(X), bf16(E)
    left = np.flatnonzero(~masked)
    target = rng.integers(0, len(left), T).astype(np.int32)
    R, tol = cross_entropy(X[:, 1:], E[left, 1:], target)
    loss, row, lse, dX, dE = ppu.ppu_head_xent(Xt.cuda(), Et.cuda(), *on_device(left[target].astype(np.int32)))
    assert not dX[:, 0].any() and not dE[torch.from_numpy(masked).cuda()].any()
    check((loss, row, lse, dX[:, 1:], dE[torch.from_numpy(left).cuda(), 1:]), R, tol)


@gpu
@pytest.mark.parametrize("T,V", [(260, 700), (24, 33000), (24, 70000)])
def test_a_row_with_an_infinite_logit_leaves_the_others_alone(T, V):
    """Its own loss is not finite, nor is their sum; the other rows keep their bits."""
    import torch
    from paper_2509_22418_b200 import ppu
    _, Xt, _, Et, _, target = make(T, 64, V, seed=V)
    tt, = on_device(target)
    ids = torch.stack([tt, (tt + 5) % V, (tt + 1) % V], 1).contiguous()
    z = torch.randn(T, 3, device="cuda")
    Xt[:, 0], Et[:, 0] = 0, 0
    Et[17, 0] = 100.0
    bad = Xt.clone()
    bad[5, 0] = 3e38
    rest = torch.arange(T, device="cuda") != 5
    for call in (lambda x: ppu.ppu_head_xent(x, Et, tt), lambda x: ppu.ppu_head_distill(x, Et, ids, z)):
        ref, got = call(Xt), call(bad)
        assert not bool(torch.isfinite(got[0])) and not bool(torch.isfinite(got[1][5])) and not bool(torch.isfinite(got[2][5]))
        for i in (1, 2, 3):
            assert torch.equal(got[i][rest], ref[i][rest])


@gpu
def test_calls_from_several_threads():
    """Each host thread on a stream and inputs of its own."""
    import torch
    from paper_2509_22418_b200 import ppu
    jobs = []
    for i in range(4):
        _, Xt, _, Et, _, target = make(200 + 57 * i, 72, 1003 + 300 * i, seed=i)
        tt, = on_device(target)
        r, g = torch.randn(len(target), 72, device="cuda"), torch.ones(72, device="cuda")

        def work(Xt=Xt, Et=Et, tt=tt, r=r, g=g):
            out = ppu.ppu_head_xent(Xt, Et, tt)
            r_out, h, stats = ppu.ppu_norm_gate_fwd(Xt, r, g, g)
            return out + (r_out, h) + ppu.ppu_norm_gate_bwd(out[3], r, Xt, r_out, stats, g, g)[:2]
        jobs.append(work)
    want = [job() for job in jobs]
    torch.cuda.synchronize()
    wrong, ready = [], threading.Barrier(len(jobs))

    def thread(i):
        try:
            stream = torch.cuda.Stream()
            ready.wait(60)
            for _ in range(30):
                with torch.cuda.stream(stream):
                    got = jobs[i]()
                with pytest.raises(ppu.PpuError, match="target"):      # (an error is its own thread's)
                    ppu.ppu_head_xent(got[3], got[4], got[1])
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                    wrong.append(i)
        except BaseException as e:
            wrong.append(e)
    threads = [threading.Thread(target=thread, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


@gpu
def test_captured_call_between_joined_streams():
    """Operands written on two other streams, results read on one of them, in one captured graph."""
    import torch
    from paper_2509_22418_b200 import ppu
    data = [make(300, 136, 2501, seed=s) for s in (1, 2)]
    data = [(x, e, *on_device(t)) for _, x, _, e, _, t in data]
    X, E, t = (torch.empty_like(a) for a in data[0])
    src = [a.clone() for a in data[0]]
    want = [ppu.ppu_head_xent(*d) for d in data]
    s1, s2, graph = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        cur = torch.cuda.current_stream()
        for s in (s1, s2):
            s.wait_stream(cur)
        with torch.cuda.stream(s1):
            X.copy_(src[0])
            t.copy_(src[2])
            t.add_(0)
        with torch.cuda.stream(s2):
            E.copy_(src[1])
            E.mul_(1)
        for s in (s1, s2):
            cur.wait_stream(s)
        out = ppu.ppu_head_xent(X, E, t)
        s1.wait_stream(cur)
        with torch.cuda.stream(s1):
            twice = out[3] * 2
        cur.wait_stream(s1)
    for i in (1, 0, 1):
        for a, b in zip(src, data[i]):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[i])) and torch.equal(twice, want[i][3] * 2)


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


@gpu
@pytest.mark.parametrize("grad", [True, False, "x", "e"])
@pytest.mark.parametrize("T,d,V,k,chunk", [(300, 72, 1003, 9, 0), (700, 72, 1003, 9, 256), (24, 64, 33000, 64, 0), (3000, 72, 1003, 3, 0), (24, 40, 70000, 128, 0)])
def test_whatever_the_workspace_held(T, d, V, k, chunk, grad):
    """Workspaces of all ones (NaN) and of zeros: the same bits."""
    import torch
    from paper_2509_22418_b200 import ppu
    rng, Xt, _, Et, _, target = make(T, d, V, seed=T)
    ids, z = teacher(rng, T, V, k, target, True)
    target[::3] = -1
    tt, it, zt = on_device(target, ids, z)
    grads = ppu._grads(grad)
    for n, call in ((1, lambda ws: ppu.ppu_head_xent(Xt, Et, tt, grad=grad, chunk_rows=chunk, workspace=ws)),
                    (k, lambda ws: ppu.ppu_head_distill(Xt, Et, it, zt, grad=grad, chunk_rows=chunk, workspace=ws))):
        size = ppu.ppu_head_query_bytes(T, d, V, grads=grads, chunk_rows=chunk, k=n)
        a, b = (call(torch.full((size,), fill, dtype=torch.uint8, device="cuda")) for fill in (0, 255))
        assert all(x is y or torch.equal(x, y) for x, y in zip(a, b))


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
