"""The front of a decoder's step as it is used: tokens through the embedding, a QKV product, the norms and rotation of queries and keys and
attention, the gradients back to the table (on top of the one that a tied head has left) and to the projections, and the projections'
orthogonalised update; also captured and replayed.

The chain rounds to bf16 at the hidden states, the products, the rotated heads, the probabilities, the attention's output and each of their gradients: about ten
roundings of at most 2^-8 (root mean square 2^-8 / sqrt(3) at most) on the way to a gradient, of which none is multiplied by more than a few: the
framework's gate of 2e-2 in relative l2 for gradients of a step, and for its results."""
import numpy as np
import pytest

from test_orthogonalize import near

pytestmark = pytest.mark.gpu


def make(B=3, S=130, heads=4, dh=64, V=501, seed=0):
    import torch
    g = torch.Generator(device="cpu").manual_seed(seed)
    d, T = heads * dh, B * S
    t = dict(ids=torch.randint(0, V, (T,), generator=g).int(), E=torch.randn(V, d, generator=g).bfloat16(), W=(torch.randn(3 * d, d, generator=g) / d ** 0.5).bfloat16(),
             qg=1 + 0.2 * torch.randn(dh, generator=g), kg=1 + 0.2 * torch.randn(dh, generator=g), dU=torch.randn(T, d, generator=g).bfloat16(),
             head=0.1 * torch.randn(V, d, generator=g), m=torch.randn(3, d, d, generator=g))
    t["ids"][5::17] = -1
    return dict(B=B, S=S, heads=heads, dh=dh, V=V, d=d), {k: v.cuda() for k, v in t.items()}


def step(ppu, c, t):
    import torch
    n = c["heads"]
    r = ppu.ppu_embed_fwd(t["ids"], t["E"], scale=0.5)
    h = r.bfloat16()
    raw = h @ t["W"].t()
    kw = dict(q_gain=t["qg"], k_gain=t["kg"], seq=c["S"], rope_base=1e4)
    qkv = ppu.ppu_qk_norm_fwd(raw, n, n, n, **kw)
    U, lse = ppu.ppu_attention_fwd(qkv, c["B"], c["S"], n, c["dh"])
    dqkv = ppu.ppu_attention_bwd(qkv, U, lse, t["dU"], c["B"], c["S"], n, c["dh"])
    draw, dqg, dkg = ppu.ppu_qk_norm_bwd(dqkv, raw, n, n, n, in_place=True, **kw)
    dW = (draw.float().t() @ h.float()).view(3, c["d"], c["d"])
    dE = ppu.ppu_embed_bwd(t["ids"], draw @ t["W"], c["V"], scale=0.5, add=t["head"])
    O, m = ppu.ppu_orthogonalize(dW, momentum=t["m"])
    return dict(U=U, dqg=dqg, dkg=dkg, dW=dW, dE=dE, O=O, m=m)


def reference(c, t):
    """The same in 64 bits, by automatic differentiation of its own formulas."""
    import torch
    x = {k: v.double().cpu() if v.is_floating_point() else v.cpu() for k, v in t.items()}
    leaves = {k: x[k].requires_grad_() for k in ("E", "W", "qg", "kg")}
    B, S, n, dh, d = c["B"], c["S"], c["heads"], c["dh"], c["d"]
    there = (x["ids"] >= 0).double()[:, None]
    h = 0.5 * leaves["E"][x["ids"].clamp(min=0).long()] * there
    q, k, v = (h @ leaves["W"].t()).view(B, S, 3, n, dh).unbind(2)
    angle = torch.arange(S, dtype=torch.float64)[:, None] * 1e4 ** (-torch.arange(0, dh, 2, dtype=torch.float64) / dh)
    turn = torch.polar(torch.ones_like(angle), angle)[None, :, None]

    def head(a, gain):
        a = a * (a.square().mean(-1, keepdim=True) + float(np.float32(1e-6))).rsqrt() * gain
        return torch.view_as_real(torch.view_as_complex(a.reshape(B, S, n, dh // 2, 2).contiguous()) * turn).flatten(-2)
    s = torch.einsum("bshe,bthe->bhst", head(q, leaves["qg"]), head(k, leaves["kg"])) / dh ** 0.5
    p = torch.softmax(s.masked_fill(torch.ones(S, S).triu(1).bool(), -torch.inf), -1)
    U = torch.einsum("bhst,bthe->bshe", p, v).reshape(B * S, d)
    g = torch.autograd.grad((U * x["dU"]).sum(), list(leaves.values()))
    out = dict(zip(("dE", "dW", "dqg", "dkg"), g))
    return out | {"U": U.detach(), "dE": out["dE"] + x["head"], "dW": out["dW"].view(3, d, d)}


@pytest.mark.parametrize("B,S,heads,dh", [(3, 130, 4, 64), (1, 257, 2, 128)])
def test_front_of_a_step(B, S, heads, dh):
    from paper_2509_22418_b200 import ppu
    c, t = make(B, S, heads, dh)
    got, want = step(ppu, c, t), reference(c, t)
    for name, w in want.items():
        g = got[name].double().cpu()
        base = t["head"].double().cpu() if name == "dE" else 0.0
        assert float((g - w).norm()) <= 2e-2 * float((w - base).norm()), name
    # the update of the gradient that the chain has formed
    dW, m = got["dW"].double().cpu().numpy(), got["m"].double().cpu().numpy()
    beta = float(np.float32(0.95))
    assert np.abs(m - (beta * t["m"].double().cpu().numpy() + dW)).max() <= 2.0 ** -22 * np.abs(m).max()
    near(got["O"], dW + beta * m)


def test_captured_beside_eager_calls():
    import torch
    from paper_2509_22418_b200 import ppu
    c, t = make()
    ref = step(ppu, c, t)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = step(ppu, c, t)
    for _ in range(3):
        eager = step(ppu, c, t)
        graph.replay()
        torch.cuda.synchronize()
        for k in ref:
            assert torch.equal(ref[k], cap[k]) and torch.equal(ref[k], eager[k]), k


def test_calls_from_several_threads():
    """Each on a stream of its own, at once: workspaces are a call's own."""
    import threading

    import torch
    from paper_2509_22418_b200 import ppu
    c, t = make(seed=3)
    ref, bad = step(ppu, c, t), []
    torch.cuda.synchronize()

    def work():
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(4):
                    got = step(ppu, c, t)
                    torch.cuda.current_stream().synchronize()
                    bad.extend(k for k in ref if not torch.equal(ref[k], got[k]))
        except Exception as e:  # noqa: BLE001
            bad.append(repr(e))
    threads = [threading.Thread(target=work) for _ in range(3)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not bad, bad
