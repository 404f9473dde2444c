"""The top of a decoder as it is used: a block's output through its norm, gate and residual addition and the
norm before the head, the head's loss (targets, or a teacher's top logits), and the gradients back down
to the block's output, the residual stream and every parameter; also captured and replayed."""
import numpy as np
import pytest

from test_head_loss import definition, hard, mean_weights, soft, teacher, tolerances
from test_norm_gate import backward, call_bwd, call_fwd, make, near

pytestmark = pytest.mark.gpu


def chain(ppu, c, t, gate_rows, E, head):
    """One pass; head(h) -> (loss, row_loss, lse, dX, dE)."""
    r_out, h, stats = call_fwd(c, t, gate_rows)
    out = head(h)
    return (r_out, h, stats) + out + call_bwd(c, dict(t, dh=out[3], dr=None), r_out, stats, gate_rows)


@pytest.mark.parametrize("kind,gate_rows", [("layer", 300), ("rms", 100), ("layer", 1), ("rms", None)])
@pytest.mark.parametrize("which", ["xent", "distill"])
def test_block_end_to_head_and_back(which, kind, gate_rows):
    import torch
    from paper_2509_22418_b200 import ppu
    T, d, V, k = 300, 136, 1003, 9
    c, t, n, v, gate, groups = make(T, d, kind, kind == "layer", gate_rows, seed=5)
    rng = np.random.default_rng(T + d)
    Et = torch.from_numpy((rng.standard_normal((V, d)) * 0.25).astype(np.float32)).bfloat16()
    E = Et.double().numpy()
    Et = Et.cuda()
    target = rng.integers(0, V, T).astype(np.int32)
    target[::7] = -1
    if which == "xent":
        ids, q, ent, there = hard(target)
        tt = torch.from_numpy(target).cuda()
        temp, head = 1.0, lambda h: ppu.ppu_head_xent(h, Et, tt)
    else:
        raw, z = teacher(rng, T, V, k, target, True)
        ids, q, ent, there = soft(raw, z, 2.0, None)
        it, zt = torch.from_numpy(raw).cuda(), torch.from_numpy(z).cuda()
        temp, head = 2.0, lambda h: ppu.ppu_head_distill(h, Et, it, zt, temperature=2.0)
    got = chain(ppu, c, t, gate_rows, Et, head)
    r_out, h, stats, loss, row, lse, dX, dE = got[:8]
    grads = dict(zip(("dy", "dr", "dg1", "db1", "dg2", "db2", "dgate"), got[8:]))
    # the head at the hidden states it was given
    H = h.double().cpu().numpy()
    w = mean_weights(there)
    R = definition(H, E, ids, q, ent, w, temp)
    tol = tolerances(H, E, q, w, temp, R, ent)
    if which == "distill":                 # the teacher's q in fp32: 64 roundings of its relative size, generously counted
        tol["dX"] += (np.abs(w) * R["Q"] * 2.0 ** -17)[:, None] * np.abs(E).max(0)[None]
        tol["loss"] += 2.0 ** -17 * (np.abs(w) * (np.abs(ent) + R["Q"] * (np.abs(R["lse"]) + np.abs(R["s"]).max(1)))).sum()
    near(dX, R["dX"], tol["dX"], "dX")
    near(loss, np.float64(R["loss"]), tol["loss"], "loss")
    # and its gradient, in 64 bits, on through the norms: the kernels had the rounded one, within tol of it
    G, gtol = backward(c, n["y"], r_out.double().cpu().numpy(), stats.double().cpu().numpy(), R["dX"], np.zeros((T, d)), v, gate, groups, e_dh=tol["dX"])
    for name in ("dy", "dr", "dg2") + (("db2",) if grads["db2"] is not None else ()):
        near(grads[name], G[name], gtol[name], name)
    # captured once, replayed on the same values: the same bits
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = chain(ppu, c, t, gate_rows, Et, head)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(a is b or torch.equal(a, b) for a, b in zip(got, again))


def test_eager_calls_beside_a_captured_pass():
    """A captured pass and eager ones of the same operands in turn, each with its own workspace."""
    import torch
    from paper_2509_22418_b200 import ppu
    c, t, *_ = make(257, 264, "layer", True, 257, seed=8)
    E = torch.randn(777, 264, device="cuda").bfloat16() * 0.1
    target = torch.randint(0, 777, (257,), device="cuda", dtype=torch.int32)
    head = lambda h: ppu.ppu_head_xent(h, E, target)  # noqa: E731
    ref = chain(ppu, c, t, 257, E, head)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = chain(ppu, c, t, 257, E, head)
    for _ in range(3):
        eager = chain(ppu, c, t, 257, E, head)
        graph.replay()
        more = chain(ppu, c, t, 257, E, head)
        torch.cuda.synchronize()
        for a, b, x, y in zip(ref, cap, eager, more):
            assert torch.equal(a, b) and torch.equal(a, x) and torch.equal(a, y)


@pytest.mark.parametrize("kind,gate_rows", [("layer", 300), ("rms", 100), ("layer", 1), ("rms", None)])
def test_gradients_of_every_parameter_below_the_head(kind, gate_rows):
    """The same chain with a cross entropy: the first norm's gain and shift and the gate too."""
    import torch
    from paper_2509_22418_b200 import ppu
    T, d, V = 300, 136, 1003
    c, t, n, v, gate, groups = make(T, d, kind, kind == "layer", gate_rows, seed=6)
    rng = np.random.default_rng(3)
    Et = torch.from_numpy((rng.standard_normal((V, d)) * 0.25).astype(np.float32)).bfloat16().cuda()
    E = Et.double().cpu().numpy()
    target = rng.integers(0, V, T).astype(np.int32)
    target[::7] = -1
    tt = torch.from_numpy(target).cuda()
    got = chain(ppu, c, t, gate_rows, Et, lambda h: ppu.ppu_head_xent(h, Et, tt))
    r_out, h, stats = got[:3]
    H = h.double().cpu().numpy()
    ids, q, ent, there = hard(target)
    w = mean_weights(there)
    R = definition(H, E, ids, q, ent, w, 1.0)
    tol = tolerances(H, E, q, w, 1.0, R, ent)
    G, gtol = backward(c, n["y"], r_out.double().cpu().numpy(), stats.double().cpu().numpy(), R["dX"], np.zeros((T, d)), v, gate, groups, e_dh=tol["dX"])
    for name, x in zip(("dy", "dr", "dg1", "db1", "dg2", "db2", "dgate"), got[8:]):
        if x is not None:
            near(x, G[name], gtol[name], name)
