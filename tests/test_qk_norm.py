"""Norms of query and key heads with the rotation by position (ppu_qk_norm_fwd / _bwd) against their definition in 64 bits, element by element.

Tolerances: u = 2^-24 (fp32, half a step).  A sum over a head is at most 8 additions in a thread and 5 between threads: with the products around it
within S = 24 u of the sum of magnitudes.  A sine or cosine: a fraction of a turn rounded to fp32 (at most 1/2: pi u), the library's 2 ulp (4 u) and
the product with the frequency in 64 bits: A = 8 u absolute.  A gain's gradient is a sum over all tokens and, where it is shared, heads: n terms in some
order within n u of the sum of magnitudes (n + 4 with the products).  bf16 results are rounded once, half a step 2^-8."""
import ctypes as C
import math

import numpy as np
import pytest

gpu = pytest.mark.gpu
U, BF = 2.0 ** -24, 2.0 ** -8
S, A = 24 * U, 8 * U


def mean(x):
    return x.mean(-1, keepdims=True)


def pairs_of(c):
    """Columns (a, b) of each pair, and their inverse frequencies."""
    r = c["rot"]
    i = np.arange(r // 2)
    f = c["freq"] if c.get("freq") is not None else c["base"] ** (-2.0 * i / max(r, 1))
    return (2 * i, 2 * i + 1, f) if c["pairs"] == "adjacent" else (i, i + r // 2, f)


def turn(x, c, pos, back=False, err=None):
    """x [T, heads, dh] turned by position; the error that x's and the angles' make."""
    a, b, f = pairs_of(c)
    angle = pos.astype(np.float64)[:, None, None] * f
    co, si = np.cos(angle), np.sin(angle) * (-1 if back else 1)
    out = x.copy()
    out[..., a], out[..., b] = x[..., a] * co - x[..., b] * si, x[..., a] * si + x[..., b] * co
    e = np.zeros_like(x) if err is None else err.copy()
    size, both = np.abs(x[..., a]) + np.abs(x[..., b]), e[..., a] * np.abs(co) + e[..., b] * np.abs(si)
    other = e[..., a] * np.abs(si) + e[..., b] * np.abs(co)
    e[..., a], e[..., b] = both + (A + 3 * U) * size, other + (A + 3 * U) * size
    return out, e


def hats(x, c):
    """xh, rstd; error of xh, relative error of rstd."""
    m = mean(x) if c["kind"] == "layer" else np.zeros_like(x[..., :1])
    y = x - m
    rstd = 1.0 / np.sqrt(mean(y * y) + c["eps"])
    xh = y * rstd
    own = rstd * S * mean(np.abs(x)) + U * np.abs(xh) if c["kind"] == "layer" else np.zeros_like(x)     # the mean's error, and its being taken off
    rel = mean(2 * own * np.abs(xh)) + mean(own ** 2) + S + 4 * U      # half of the sum of squares' relative error twice over, root, quotient
    return xh, rstd, own + np.abs(xh) * (rel + 2 * U), rel


def split(x, c, T):
    h = c["nq"] + c["nk"]
    x = x.reshape(T, -1, c["dh"])
    return x[:, :h], x[:, h:]


def gains(n, c):
    out = []
    for name, heads in (("q_gain", c["nq"]), ("k_gain", c["nk"])):
        g = n[name]
        out.append(np.ones((heads, c["dh"])) if g is None else np.broadcast_to(g, (heads, c["dh"])))
    return np.concatenate(out)


def forward(n, c, pos):
    T = len(pos)
    x, v = split(n["qkv"], c, T)
    g = gains(n, c)
    xh, _, e, _ = hats(x, c)
    y, e = turn(xh * g, c, pos, err=e * np.abs(g) + 2 * U * np.abs(xh * g))
    return np.concatenate([y, v], 1).reshape(T, -1), np.concatenate([e * (1 + BF) + BF * np.abs(y), 0 * v], 1).reshape(T, -1)


def backward(n, c, pos):
    T = len(pos)
    x, _ = split(n["qkv"], c, T)
    dy, dv = split(n["dout"], c, T)
    g = gains(n, c)
    xh, rstd, e_xh, rel = hats(x, c)
    z, e_z = turn(dy, c, pos, back=True)
    w, e_w = z * g, e_z * np.abs(g) + U * np.abs(z * g)
    ab = np.abs
    dot, e_dot = mean(w * xh), mean(e_w * ab(xh) + ab(w) * e_xh) + (S + 4 * U) * mean(ab(w * xh))
    inner = w - xh * dot
    e_in = e_w + e_xh * ab(dot) + ab(xh) * e_dot + 4 * U * (ab(w) + ab(xh * dot))
    if c["kind"] == "layer":
        inner = inner - mean(w)
        e_in = e_in + mean(e_w) + (S + 4 * U) * mean(ab(w))
    dx = rstd * inner
    e_dx = rstd * e_in + (rel + 4 * U) * ab(dx)
    dg, e_dg = z * xh, e_z * ab(xh) + ab(z) * e_xh + 4 * U * ab(z * xh)
    out = {"dqkv": (np.concatenate([dx, dv], 1).reshape(T, -1), np.concatenate([e_dx * (1 + BF) + BF * ab(dx), 0 * dv], 1).reshape(T, -1))}
    for name, part in (("q_gain", slice(0, c["nq"])), ("k_gain", slice(c["nq"], None))):
        if n[name] is None:
            out["d" + name] = None
            continue
        axes = (0,) if n[name].ndim == 2 else (0, 1)
        terms = T * (1 if n[name].ndim == 2 else dg[:, part].shape[1])
        out["d" + name] = dg[:, part].sum(axes), e_dg[:, part].sum(axes) + terms * U * ab(dg[:, part]).sum(axes) + 1e-37
    return out


def make(T, nq, nk, nv, dh, kind="rms", pairs="adjacent", rot=None, gain="shared", seed=0, eps=1e-6, base=1e4, size=1.0, far=False, shift=0.0, freq=False):
    import torch
    rng = np.random.default_rng(seed + T + 10 * nq + 100 * dh)
    f = lambda a: torch.from_numpy(np.asarray(a, dtype=np.float32))  # noqa: E731
    shape = {"shared": lambda h: (dh,), "heads": lambda h: (h, dh)}
    t = dict(qkv=(f(rng.standard_normal((T, (nq + nk + nv) * dh)) * size + shift)).bfloat16(), dout=f(rng.standard_normal((T, (nq + nk + nv) * dh)) * 0.1).bfloat16())
    for name, h in (("q_gain", nq), ("k_gain", nk)):
        t[name] = None if gain is None else f(1 + 0.3 * rng.standard_normal(shape[gain](h)))
    pos = rng.integers(0, 1 << 20, T) if far else np.arange(T)
    c = dict(nq=nq, nk=nk, nv=nv, dh=dh, kind=kind, pairs=pairs, rot=dh if rot is None else rot, eps=float(np.float32(eps)), base=float(np.float32(base)))
    t["inv_freq"] = f(0.5 ** np.arange(c["rot"] // 2)) if freq else None
    c["freq"] = t["inv_freq"].double().numpy() if freq else None
    t["positions"] = torch.from_numpy(pos.astype(np.int32)) if far else None
    n = {k: None if x is None else x.double().numpy() for k, x in t.items()}
    return c, {k: None if x is None else x.cuda() for k, x in t.items()}, n, pos


def more(c, t):
    return dict(q_gain=t["q_gain"], k_gain=t["k_gain"], positions=t["positions"], kind=c["kind"], eps=c["eps"], rope_base=c["base"], inv_freq=t["inv_freq"],
                rot_dim=c["rot"], pairs=c["pairs"])


def call_fwd(c, t, **kw):
    from paper_2509_22418_b200 import ppu
    return ppu.ppu_qk_norm_fwd(t["qkv"], c["nq"], c["nk"], c["nv"], **{**more(c, t), **kw})


def call_bwd(c, t, **kw):
    from paper_2509_22418_b200 import ppu
    return ppu.ppu_qk_norm_bwd(t["dout"], t["qkv"], c["nq"], c["nk"], c["nv"], **{**more(c, t), **kw})


def near(got, want, tol, name=""):
    g = got.detach().double().cpu().numpy()
    err = np.abs(g - want)
    assert g.shape == want.shape and np.all(err <= tol + 1e-37), (name, float(err.max()), float((err / (tol + 1e-37)).max()))


def check(c, t, n, pos, **kw):
    near(call_fwd(c, t, **kw), *forward(n, c, pos), "out")
    got = dict(zip(("dqkv", "dq_gain", "dk_gain"), call_bwd(c, t, **kw)))
    for name, want in backward(n, c, pos).items():
        if want is None:
            assert got[name] is None
        else:
            near(got[name], *want, name)


CASES = [
    # T, nq, nk, nv, dh, rot
    (1, 1, 1, 1, 8, 8), (1, 32, 8, 8, 128, 128), (3, 2, 1, 0, 16, 8), (17, 3, 3, 3, 24, 16), (100, 4, 2, 2, 32, 32), (65, 5, 5, 5, 40, 0), (130, 7, 1, 1, 64, 64),
    (333, 6, 2, 2, 80, 32), (50, 12, 12, 12, 96, 96), (257, 16, 16, 16, 128, 128), (70, 9, 3, 0, 160, 64), (41, 8, 4, 4, 192, 192), (29, 3, 2, 1, 256, 256),
    (1000, 1, 1, 1, 16, 16), (5000, 2, 2, 0, 8, 8), (2, 100, 28, 28, 64, 16), (600, 0, 4, 4, 64, 64), (90, 6, 0, 0, 112, 112), (3000, 1, 0, 0, 256, 256),
]


@gpu
@pytest.mark.parametrize("kind,pairs,gain", [("rms", "adjacent", "shared"), ("rms", "halves", "heads"), ("layer", "halves", "shared"), ("layer", "adjacent", "heads"),
                                             ("rms", "halves", None)])
@pytest.mark.parametrize("T,nq,nk,nv,dh,rot", CASES)
def test_against_the_definition(T, nq, nk, nv, dh, rot, kind, pairs, gain):
    check(*make(T, nq, nk, nv, dh, kind, pairs, rot, gain, far=T % 2 == 1))


@gpu
def test_positions():
    """Sequences one after another, negative and the largest positions, a base and frequencies of one's own."""
    import torch
    c, t, n, pos = make(500, 4, 2, 2, 64)
    near(call_fwd(c, t, seq=37), *forward(n, c, pos % 37), "seq")
    t["positions"] = torch.from_numpy((pos % 37).astype(np.int32)).cuda()
    assert torch.equal(call_fwd(c, t), call_fwd(c, dict(t, positions=None), seq=37))
    ends = np.array([2 ** 31 - 1, -2 ** 31, -1, 2 ** 31 - 2, 1 << 30] * 100)
    t["positions"] = torch.from_numpy(ends.astype(np.int32)).cuda()
    check(c, t, n, ends)
    for kw in (dict(base=5e5), dict(base=0.5), dict(freq=True)):
        check(*make(300, 4, 2, 2, 64, far=True, **kw))


@gpu
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_heads_far_from_the_ordinary(kind):
    """A mean a hundred times the deviation, tiny and large heads, heads of zeros and constant ones, no eps."""
    import torch
    check(*make(64, 4, 2, 2, 128, kind, shift=100.0))
    check(*make(64, 4, 2, 2, 128, kind, size=1e-6, eps=1e-12))
    check(*make(64, 4, 2, 2, 128, kind, size=1e8))
    check(*make(77, 3, 2, 0, 80, kind, eps=0.0, rot=16, pairs="halves"))
    c, t, n, pos = make(30, 2, 2, 2, 64, kind)
    t["qkv"][3] = 0.0
    t["qkv"][4] = 2.0
    n["qkv"] = t["qkv"].double().cpu().numpy()
    check(c, t, n, pos)


@gpu
def test_a_row_of_nan_leaves_the_others_alone():
    import torch
    c, t, n, pos = make(60, 4, 2, 2, 64)
    clean, grads = call_fwd(c, t), call_bwd(c, t)
    t["qkv"][11, 70] = float("nan")          # one value of the second query head
    t["qkv"][12, 0] = float("inf")
    got, dg = call_fwd(c, t), call_bwd(c, t)
    keep = [i for i in range(60) if i not in (11, 12)]
    assert torch.equal(got[keep], clean[keep]) and torch.equal(dg[0][keep], grads[0][keep])
    assert torch.isnan(got[11, 64:128].float()).all() and torch.equal(got[11, 128:], clean[11, 128:]) and torch.equal(got[11, :64], clean[11, :64])
    assert torch.isnan(dg[1]).any() and torch.equal(dg[2], grads[2])


@gpu
@pytest.mark.parametrize("pairs", ["adjacent", "halves"])
def test_in_place_and_strided(pairs):
    import torch
    c, t, n, pos = make(200, 4, 2, 2, 48, "layer", pairs, rot=32, gain="heads")
    out, grads = call_fwd(c, t), call_bwd(c, t)
    wide = torch.full((202, 400), 7.0, dtype=torch.bfloat16, device="cuda")
    view = wide[1:201, 8:392]
    view.copy_(t["qkv"])
    assert torch.equal(call_fwd(c, dict(t, qkv=view)), out)
    dwide = torch.full((200, 392), float("nan"), dtype=torch.bfloat16, device="cuda")
    dwide[:, :384] = t["dout"]
    dview = dwide[:, :384]
    for a, b in zip(call_bwd(c, dict(t, qkv=view, dout=dview)), grads):
        assert torch.equal(a, b)
    got = call_bwd(c, dict(t, dout=dview), in_place=True)
    assert got[0] is dview and all(torch.equal(a, b) for a, b in zip(got, grads)) and torch.isnan(dwide[:, 384:].float()).all()
    assert call_fwd(c, dict(t, qkv=view), in_place=True) is view and torch.equal(view, out)
    view.fill_(7.0)
    assert bool((wide == 7.0).all())


@gpu
def test_gradients_against_differences():
    """Central differences of sum(y dout) in 64 bits of the definition, along directions of x and of the gains."""
    c, t, n, pos = make(20, 3, 1, 1, 32, "layer", "halves", rot=16, gain="heads", far=True)
    got = [g.double().cpu().numpy() for g in call_bwd(c, t)]
    rng = np.random.default_rng(5)
    f = lambda m: float((forward(m, c, pos)[0] * n["dout"]).sum())  # noqa: E731
    for name, g in zip(("qkv", "q_gain", "k_gain"), got):
        d = rng.standard_normal(n[name].shape)
        h = 1e-4
        num = (f({**n, name: n[name] + h * d}) - f({**n, name: n[name] - h * d})) / (2 * h)
        assert abs(num - float((g * d).sum())) <= BF * float(np.abs(g * d).sum()) + 1e-5 * abs(num)


@gpu
@pytest.mark.parametrize("T", [1, 700])
def test_captured_streamed_and_repeated_calls_have_the_same_bits(T):
    import torch
    from paper_2509_22418_b200 import ppu
    c, t, n, pos = make(T, 8, 4, 4, 64, far=True)
    ref = (call_fwd(c, t),) + call_bwd(c, t)
    nb = ppu.ppu_qk_norm_query_bytes(T, 8, 4, 4, 64)
    for fill in (0, 255):
        got = call_bwd(c, t, workspace=torch.full((nb,), fill, dtype=torch.uint8, device="cuda"))
        assert all(torch.equal(a, b) for a, b in zip(got, ref[1:]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = (call_fwd(c, t),) + call_bwd(c, t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        graph.replay()
        with torch.cuda.stream(side):
            other = (call_fwd(c, t),) + call_bwd(c, t)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(x, b) for a, x, b in zip(cap, other, ref))


@gpu
def test_offsets_beyond_32_bits():
    import torch
    T = (1 << 21) + 3                          # 2.1 billion elements
    c, t, n, pos = make(3, 8, 4, 4, 64)
    last = torch.arange(T - 3, T, dtype=torch.int32, device="cuda")
    small = dict(t, positions=last)
    x, g = (torch.zeros((T, 1024), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x[-3:], g[-3:] = t["qkv"], t["dout"]
    out, ref = call_fwd(c, dict(t, qkv=x)), call_fwd(c, small)
    assert torch.equal(out[-3:], ref) and not out[:-3].any()
    del out
    got, want = call_bwd(c, dict(t, qkv=x, dout=g), in_place=True), call_bwd(c, small)
    assert torch.equal(got[0][-3:], want[0]) and not got[0][:-3].any()
    for a, b in zip(got[1:], want[1:]):
        assert torch.allclose(a, b, rtol=1e-5, atol=1e-6)      # (the same three terms, joined at other places)


@gpu
def test_no_rows():
    import torch
    c, t, n, pos = make(4, 2, 1, 1, 16)
    z = dict(t, qkv=t["qkv"][:0], dout=t["dout"][:0])
    assert call_fwd(c, z).shape == (0, 64)
    got = call_bwd(c, z)
    assert got[0].shape == (0, 64) and not got[1].any() and not got[2].any()


@gpu
def test_writing_in_place_is_seen_by_autograd():
    import torch
    c, t, n, pos = make(4, 2, 1, 1, 16)
    x = t["qkv"].clone()
    before = x._version
    call_fwd(c, dict(t, qkv=x), in_place=True)
    assert x._version > before
    leaf = t["qkv"].clone().requires_grad_()
    from paper_2509_22418_b200 import ppu
    with pytest.raises(ppu.PpuError):
        call_fwd(c, dict(t, qkv=leaf), in_place=True)
    with pytest.raises(ppu.PpuError):
        call_bwd(c, dict(t, dout=leaf), in_place=True)
    with torch.no_grad():
        call_fwd(c, dict(t, qkv=leaf), in_place=True)


# ---- refusals ----------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def ppu():
    from paper_2509_22418_b200 import build, ppu as mod
    build.build()
    return mod


F = ["x", "ldx", "qg", "kg", "each", "pos", "seq", "kind", "eps", "base", "freq", "rot", "pairs", "out", "ldo", "T", "nq", "nk", "nv", "dh", "st"]
B = ["dy", "ldy", "x", "ldx", "qg", "kg", "each", "pos", "seq", "kind", "eps", "base", "freq", "rot", "pairs", "out", "ldo", "dqg", "dkg", "T", "nq", "nk", "nv", "dh", "ws",
     "nb", "st"]


def _call(fn, names, **change):
    buf = (C.c_uint8 * 65536)()
    base = (C.addressof(buf) + 255) & ~255
    a = {n: C.c_void_p(base) for n in names}
    a.update({n: C.c_int64(64) for n in ("ldx", "ldy", "ldo")}, each=0, pos=None, seq=0, kind=1, eps=C.c_float(1e-6), base=C.c_float(1e4), freq=None, rot=16, pairs=0, T=4, nq=2,
             nk=1, nv=1, dh=16, st=None, nb=C.c_size_t(1 << 40), out=C.c_void_p(base + 8192))
    for n, x in change.items():
        a[n] = C.c_void_p(base + 8) if x == "odd" else C.c_void_p(base + 2) if x == "odder" else C.c_void_p(base) if x == "there" else x
    return fn(*[a[n] for n in names])


BOTH = [(dict(x=None), -1), (dict(out=None), -1), (dict(dh=12), -2), (dict(dh=264), -2), (dict(dh=0), -1), (dict(T=-1), -1), (dict(T=(1 << 24) + 1), -2), (dict(nq=-1), -1),
        (dict(nq=0, nk=0), -1), (dict(nq=5000), -2), (dict(kind=2), -1), (dict(pairs=2), -1), (dict(rot=20), -2), (dict(rot=12), -2), (dict(rot=-8), -2), (dict(eps=C.c_float(-1)), -1),
        (dict(eps=C.c_float(math.nan)), -1), (dict(base=C.c_float(0)), -1), (dict(base=C.c_float(math.inf)), -1), (dict(base=C.c_float(math.nan)), -1), (dict(seq=-1), -1),
        (dict(ldx=C.c_int64(56)), -1), (dict(ldo=C.c_int64(68)), -1), (dict(x="odd"), -1), (dict(out="odd"), -1), (dict(qg="odd"), -1), (dict(pos="odder"), -1)]


@pytest.mark.parametrize("change,code", BOTH + [(dict(out="there", ldo=C.c_int64(72)), -1)])
def test_forward_refuses(ppu, change, code):
    assert _call(ppu.lib().ppu_qk_norm_fwd, F, **change) == code


@pytest.mark.parametrize("change,code", BOTH + [(dict(dy=None), -1), (dict(ws=None), -1), (dict(nb=C.c_size_t(8)), -4), (dict(ws="odd"), -1), (dict(qg=None), -1),
                                                (dict(kg=None), -1), (dict(ldy=C.c_int64(60)), -1), (dict(out="there", ldo=C.c_int64(72)), -1)])
def test_backward_refuses(ppu, change, code):
    assert _call(ppu.lib().ppu_qk_norm_bwd, B, **change) == code


def test_workspace_sizes(ppu):
    assert ppu.ppu_qk_norm_query_bytes(0, 2, 2, 2, 64) == 0
    for args in ((1, 1, 1, 1, 8), (8192, 16, 16, 16, 128), (1 << 24, 32, 8, 8, 256)):
        assert 0 < ppu.ppu_qk_norm_query_bytes(*args) <= ppu.ppu_qk_norm_query_bytes(*args, gain_per_head=True) + 8 * 148 * 2048 <= 1 << 26
    for bad in ((-1, 1, 1, 1, 8), (1, 0, 0, 1, 8), (1, 1, 1, 1, 12)):
        with pytest.raises(ppu.PpuError):
            ppu.ppu_qk_norm_query_bytes(*bad)


def test_words_and_tensors_are_checked(ppu):
    import torch
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    for call in (lambda: ppu.ppu_qk_norm_fwd(x, 2, 1, 1), lambda: ppu.ppu_qk_norm_bwd(x, x, 2, 1, 1), lambda: ppu.ppu_qk_norm_fwd(x, 2, 1, 1, kind="batch"),
                 lambda: ppu.ppu_qk_norm_fwd(x, 2, 1, 1, pairs="both")):
        with pytest.raises(ppu.PpuError):
            call()


@gpu
def test_device_tensors_are_checked():
    import torch
    from paper_2509_22418_b200 import ppu
    c = dict(device="cuda")
    x, g = torch.zeros(4, 64, dtype=torch.bfloat16, **c), torch.ones(16, **c)
    for args, kw in (((x.float(), 2, 1, 1), {}), ((x, 2, 1, 2), {}), ((x, 0, 0, 4), {}), ((x, -1, 4, 1), {}), ((x.t(), 2, 1, 1), {}), ((x, 2, 1, 1), dict(q_gain=g[:8])),
                     ((x, 2, 1, 1), dict(q_gain=g, k_gain=torch.ones(1, 16, **c))), ((x, 2, 1, 1), dict(q_gain=torch.ones(3, 16, **c))), ((x, 2, 1, 1), dict(q_gain=g.double())),
                     ((x, 2, 1, 1), dict(positions=torch.zeros(3, dtype=torch.int32, **c))), ((x, 2, 1, 1), dict(positions=torch.zeros(4, dtype=torch.int64, **c))),
                     ((x, 2, 1, 1), dict(inv_freq=torch.ones(4, **c))), ((x, 2, 1, 1), dict(rot_dim=24)), ((x, 2, 1, 1), dict(eps=-1.0)), ((x[:, :60], 2, 1, 1), {})):
        with pytest.raises(ppu.PpuError):
            ppu.ppu_qk_norm_fwd(*args, **kw)
    for args, kw in (((x[:3], x, 2, 1, 1), {}), ((x.float(), x, 2, 1, 1), {}), ((x, x, 2, 1, 1), dict(q_gain=g, workspace=torch.zeros(8, dtype=torch.uint8, **c)))):
        with pytest.raises(ppu.PpuError):
            ppu.ppu_qk_norm_bwd(*args, **kw)
