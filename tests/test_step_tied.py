"""A decoder's step with a tied table, whole: lookup, QKV product, norms and rotation, attention, the residual stream, the head loss against the table, and back,
where the lookup's gradient is formed in the place of the one that the head loss has left; then the projections' update.  Also captured and replayed.

As in test_step_front.py: some ten roundings of at most 2^-8 to bf16 on the way to a gradient, the framework's gate of 2e-2 in relative l2; the table's sum is
rounded to bf16 once more, half a step of 2^-8 of its values."""
import numpy as np
import pytest

from test_orthogonalize import near

pytestmark = pytest.mark.gpu
SCALE = 16.0


def make(B, S, heads, dh, V, seed=0):
    import torch
    g = torch.Generator(device="cpu").manual_seed(seed)
    d, T = heads * dh, B * S
    t = dict(ids=torch.randint(0, V, (T,), generator=g).int(), E=(torch.randn(V, d, generator=g) / SCALE).bfloat16(),
             W=(torch.randn(3 * d, d, generator=g) / d ** 0.5).bfloat16(), qg=1 + 0.2 * torch.randn(dh, generator=g), kg=1 + 0.2 * torch.randn(dh, generator=g),
             m=1e-3 * torch.randn(3, d, d, generator=g))
    t["ids"][5::17] = -1
    ids = t["ids"].view(B, S)
    t["target"] = torch.cat([ids[:, 1:], torch.full((B, 1), -1)], 1).int().flatten()      # (absent tokens are no targets)
    return dict(B=B, S=S, heads=heads, dh=dh, V=V, d=d), {k: v.cuda() for k, v in t.items()}


def step(ppu, c, t):
    import torch
    n = c["heads"]
    r = ppu.ppu_embed_fwd(t["ids"], t["E"], scale=SCALE)
    h = r.bfloat16()
    raw = h @ t["W"].t()
    kw = dict(q_gain=t["qg"], k_gain=t["kg"], seq=c["S"])
    qkv = ppu.ppu_qk_norm_fwd(raw, n, n, n, **kw)
    U, lse = ppu.ppu_attention_fwd(qkv, c["B"], c["S"], n, c["dh"])
    X = (r + U.float()).bfloat16()
    loss, _, _, dX, dE = ppu.ppu_head_xent(X, t["E"], t["target"])
    head = dE.clone()
    dqkv = ppu.ppu_attention_bwd(qkv, U, lse, dX, c["B"], c["S"], n, c["dh"])
    draw, dqg, dkg = ppu.ppu_qk_norm_bwd(dqkv, raw, n, n, n, in_place=True, **kw)
    dW = (draw.float().t() @ h.float()).view(3, c["d"], c["d"])
    dr = dX.float() + (draw @ t["W"]).float()
    out = ppu.ppu_embed_bwd(t["ids"], dr, c["V"], scale=SCALE, add=dE, in_place=True)
    assert out.data_ptr() == dE.data_ptr()
    O, m = ppu.ppu_orthogonalize(dW, momentum=t["m"].clone(), in_place=True)
    return dict(loss=loss, dqg=dqg, dkg=dkg, dW=dW, head=head, dE=dE, O=O, m=m)


def reference(c, t):
    """The same in 64 bits, by automatic differentiation of its own formulas; the table's two uses apart."""
    import torch
    x = {k: v.double().cpu() if v.is_floating_point() else v.cpu() for k, v in t.items()}
    B, S, n, dh, d = c["B"], c["S"], c["heads"], c["dh"], c["d"]
    E, H, W, qg, kg = (x[k].clone().requires_grad_() for k in ("E", "E", "W", "qg", "kg"))
    r = SCALE * E[x["ids"].clamp(min=0).long()] * (x["ids"] >= 0).double()[:, None]
    q, k, v = (r @ W.t()).view(B, S, 3, n, dh).unbind(2)
    angle = torch.arange(S, dtype=torch.float64)[:, None] * 1e4 ** (-torch.arange(0, dh, 2, dtype=torch.float64) / dh)
    turn = torch.polar(torch.ones_like(angle), angle)[None, :, None]

    def head(a, gain):
        a = a * (a.square().mean(-1, keepdim=True) + float(np.float32(1e-6))).rsqrt() * gain
        return torch.view_as_real(torch.view_as_complex(a.reshape(B, S, n, dh // 2, 2).contiguous()) * turn).flatten(-2)
    s = torch.einsum("bshe,bthe->bhst", head(q, qg), head(k, kg)) / dh ** 0.5
    p = torch.softmax(s.masked_fill(torch.ones(S, S).triu(1).bool(), -torch.inf), -1)
    X = r + torch.einsum("bhst,bthe->bshe", p, v).reshape(B * S, d)
    counts = x["target"] >= 0
    logp = torch.log_softmax(X @ H.t(), -1)[counts]
    loss = -logp.gather(1, x["target"][counts].long()[:, None]).mean()
    dE, dH, dW, dqg, dkg = torch.autograd.grad(loss, [E, H, W, qg, kg])
    return dict(loss=loss.detach(), dqg=dqg, dkg=dkg, dW=dW.view(3, d, d), head=dH, dE=dE + dH)


@pytest.mark.parametrize("B,S,heads,dh,V", [(3, 130, 4, 64, 501), (1, 257, 2, 128, 1000)])
def test_a_step_with_a_tied_table(B, S, heads, dh, V):
    from paper_2509_22418_b200 import ppu
    c, t = make(B, S, heads, dh, V)
    got, want = step(ppu, c, t), reference(c, t)
    for name, w in want.items():
        assert float((got[name].double().cpu() - w).norm()) <= 2e-2 * float(w.norm()), name
    # the lookup's part of the table's gradient by itself
    part, mine = want["dE"] - want["head"], got["dE"].double().cpu() - got["head"].double().cpu()
    assert float((mine - part).norm()) <= 2e-2 * float(part.norm()) + 2.0 ** -8 * float(want["dE"].norm())
    dW, m = got["dW"].double().cpu().numpy(), got["m"].double().cpu().numpy()
    near(got["O"], dW + float(np.float32(0.95)) * m)


def test_captured_beside_eager_steps():
    import torch
    from paper_2509_22418_b200 import ppu
    c, t = make(2, 100, 4, 64, 333, seed=2)
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
