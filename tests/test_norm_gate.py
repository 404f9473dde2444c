"""The norms before and after a block with its gate and the residual scale (ppu_norm_gate_fwd / _bwd)
against their definition in 64 bits, element by element.

Tolerances: u = 2^-24 (fp32, half a step), a sum over a row is at most 8 additions in a thread, 5 in
a warp and 16 across warps, so with the products around it within S = 48 u of the sum of magnitudes;
a sum over rows is one running sum per unit and a sum over at most 2368 units by 32 warps: at most (T + 110) u
of the sum of magnitudes; bf16 results are rounded once, half a step 2^-8."""
import ctypes as C
import math

import numpy as np
import pytest

gpu = pytest.mark.gpu
U = 2.0 ** -24
S = 48 * U
BF = 2.0 ** -8


def norm(x, kind, eps):
    mean = x.mean(1, keepdims=True) if kind == "layer" else np.zeros((len(x), 1))
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    return (x - mean) * rstd, mean, rstd


def forward(c, y, r, v, gate):
    yh, m1, s1 = norm(y, c["kind"], c["eps"])
    n = yh * v["g1"] + v["b1"]
    r_out = c["scale"] * r + gate * n
    rh, m2, s2 = norm(r_out, c["kind"], c["eps"])
    return dict(yh=yh, n=n, r_out=r_out, rh=rh, h=rh * v["g2"] + v["b2"], stats=np.concatenate([m1, s1, m2, s2], 1))


def hat_error(x, x_err, xh, mean, rstd):
    """Error of (x - mean) rstd from that of x, the mean's and the deviation's sums."""
    size = np.abs(x).mean(1, keepdims=True)
    own = rstd * (x_err + S * (size + np.abs(mean)) + x_err.mean(1, keepdims=True))
    # the deviation: half the relative error of the mean square (its terms 2 own |xh|), and the root
    rel = (2 * own * np.abs(xh)).mean(1, keepdims=True) + (own ** 2).mean(1, keepdims=True) + 2 * S
    return own + np.abs(xh) * rel, rel


def backward(c, y, r_out, st, dh, dr, v, gate, groups, e_dh=0.0):
    """The definition's gradients and their tolerances; e_dh: how far the dh that was used may be from this one."""
    m1, s1, m2, s2 = (st[:, i:i + 1] for i in range(4))
    yh, rh = (y - m1) * s1, (r_out - m2) * s2
    dhat = dh * v["g2"]

    def through(dx, xh, s):
        out = dx - xh * (dx * xh).mean(1, keepdims=True)
        return s * (out - dx.mean(1, keepdims=True) if c["kind"] == "layer" else out)
    G = dr + through(dhat, rh, s2)
    dn = gate * G
    q = dn * v["g1"]
    dy = through(q, yh, s1)
    rows = G * (yh * v["g1"] + v["b1"])
    dgate = np.zeros((groups, y.shape[1]))
    np.add.at(dgate, np.arange(len(y)) // c["gate_rows"], rows)
    R = dict(dy=dy, dr=c["scale"] * G, dg1=(dn * yh).sum(0), db1=dn.sum(0), dg2=(dh * rh).sum(0), db2=dh.sum(0), dgate=dgate)
    # tolerances
    a = np.abs
    e_yh = 4 * U * s1 * (a(y) + a(m1)) + 2 * U * a(yh)
    e_rh = 4 * U * s2 * (a(r_out) + a(m2)) + 2 * U * a(rh)

    def through_error(dx, e_dx, xh, e_xh, s):
        mean = lambda z: z.mean(1, keepdims=True)  # noqa: E731
        dot = mean(a(dx * xh))
        e_dot = mean(e_dx * a(xh) + a(dx) * e_xh) + S * dot
        return s * (e_dx + S * mean(a(dx)) + mean(e_dx) + e_xh * dot + (a(xh) + e_xh) * e_dot) + 6 * U * s * (a(dx) + mean(a(dx)) + a(xh) * dot)
    e_G = 2 * U * a(dr) + through_error(dhat, 2 * U * a(dhat) + a(v["g2"]) * e_dh, rh, e_rh, s2)
    e_q = a(gate * v["g1"]) * e_G + 4 * U * a(q)
    e_dy = through_error(q, e_q, yh, e_yh, s1)
    over = (len(y) + 110) * U
    e_rows = a(yh * v["g1"] + v["b1"]) * e_G + a(G) * (a(v["g1"]) * e_yh + 6 * U * (a(yh * v["g1"]) + a(v["b1"])))
    mag_rows = a(G) * (a(yh * v["g1"]) + a(v["b1"]))        # the kernel sums G yhat and G apart
    e_gate, mag_gate = np.zeros_like(dgate), np.zeros_like(dgate)
    np.add.at(e_gate, np.arange(len(y)) // c["gate_rows"], e_rows)
    np.add.at(mag_gate, np.arange(len(y)) // c["gate_rows"], mag_rows)
    e_dn = a(gate) * e_G + 2 * U * a(dn)
    tol = dict(dy=e_dy * (1 + BF) + BF * a(dy), dr=c["scale"] * e_G + 2 * U * a(c["scale"] * G),
               dg1=(e_dn * a(yh) + a(dn) * e_yh).sum(0) + over * a(dn * yh).sum(0), db1=e_dn.sum(0) + over * a(dn).sum(0),
               dg2=(a(dh) * e_rh + e_dh * (a(rh) + e_rh)).sum(0) + over * a(dh * rh).sum(0),
               db2=(e_dh + over * a(dh)).sum(0), dgate=e_gate + over * mag_gate)
    return R, {n: t + 1e-30 for n, t in tol.items()}


def make(T, d, kind="layer", shift=True, gate_rows=None, scale=0.9, seed=0, eps=1e-5, mean=0.1):
    """gate_rows None: no gate."""
    import torch
    rng = np.random.default_rng(seed + 7 * T + d)
    f = lambda a: torch.from_numpy(np.asarray(a, dtype=np.float32))  # noqa: E731
    t = dict(y=f(rng.standard_normal((T, d)) * 0.7 + mean).bfloat16(), r=f(rng.standard_normal((T, d)) * 1.5 + mean),
             g1=f(1 + 0.2 * rng.standard_normal(d)), g2=f(1 + 0.2 * rng.standard_normal(d)),
             b1=f(0.1 * rng.standard_normal(d)) if shift else None, b2=f(0.1 * rng.standard_normal(d)) if shift else None,
             dh=f(rng.standard_normal((T, d)) * 0.05).bfloat16(), dr=f(rng.standard_normal((T, d)) * 0.05))
    groups = -(-T // gate_rows) if gate_rows else 1
    t["gate"] = f(0.5 + 0.3 * rng.standard_normal((groups, d))) if gate_rows else None
    c = dict(kind=kind, scale=float(np.float32(scale)), eps=float(np.float32(eps)), gate_rows=gate_rows or max(T, 1))
    n = {k: None if x is None else x.double().numpy() for k, x in t.items()}
    v = dict(g1=n["g1"], g2=n["g2"], b1=np.zeros(d) if n["b1"] is None else n["b1"], b2=np.zeros(d) if n["b2"] is None else n["b2"])
    gate = np.ones((T, 1)) if n["gate"] is None else n["gate"][np.arange(T) // c["gate_rows"]]
    return c, {k: None if x is None else x.cuda() for k, x in t.items()}, n, v, gate, groups


def call_fwd(c, t, gate_rows, **more):
    from paper_2509_22418_b200 import ppu
    return ppu.ppu_norm_gate_fwd(t["y"], t["r"], t["g1"], t["g2"], post_shift=t["b1"], pre_shift=t["b2"], gate=t["gate"], gate_rows=gate_rows or 0,
                                 kind=c["kind"], res_scale=c["scale"], eps=c["eps"], **more)


def call_bwd(c, t, r_out, stats, gate_rows, **more):
    from paper_2509_22418_b200 import ppu
    return ppu.ppu_norm_gate_bwd(t["dh"], t["dr"], t["y"], r_out, stats, t["g1"], t["g2"], post_shift=t["b1"], pre_shift=t["b2"], gate=t["gate"],
                                 gate_rows=gate_rows or 0, kind=c["kind"], res_scale=c["scale"], **more)


def near(got, want, tol, name):
    g = got.detach().float().cpu().numpy().astype(np.float64)
    err = np.abs(g - want)
    assert g.shape == want.shape and np.all(err <= tol), (name, float(err.max()), float((err / tol).max()))


CASES = [
    # T, d, gate_rows
    (1, 8, None), (1, 2048, 1), (2, 64, 2), (3, 72, 1), (5, 40, 2),
    (777, 64, 100),         # several units to a group, several units to a warp
    (2500, 16, 1),          # more groups than units
    (5000, 8, 3),           # the same, a last group of two rows
    (257, 136, None), (300, 256, 300), (1500, 264, 7),
    (333, 768, 64), (1001, 1032, 1), (130, 2048, 130), (400, 2056, 2), (97, 4096, 10), (1, 4096, None),
    (20000, 8, 1), (1301, 264, 1), (1640, 256, 10), (3000, 32, None), (1999, 520, 1), (350, 2104, 90), (161, 2568, None),
]


@gpu
@pytest.mark.parametrize("kind,shift", [("layer", True), ("rms", False), ("layer", False), ("rms", True)])
@pytest.mark.parametrize("T,d,gate_rows", CASES)
def test_against_the_definition(T, d, gate_rows, kind, shift):
    import torch
    c, t, n, v, gate, groups = make(T, d, kind, shift, gate_rows)
    F = forward(c, n["y"], n["r"], v, gate)
    r_out, h, stats = call_fwd(c, t, gate_rows)
    st = F["stats"]
    e_yh, rel1 = hat_error(n["y"], np.zeros_like(n["y"]), F["yh"], st[:, 0:1], st[:, 1:2])
    e_n = np.abs(v["g1"]) * e_yh + 4 * U * (np.abs(F["yh"] * v["g1"]) + np.abs(v["b1"]))
    e_r = np.abs(gate) * e_n + 4 * U * (np.abs(gate * F["n"]) + np.abs(gate * v["b1"]) + np.abs(c["scale"] * n["r"]))
    near(r_out, F["r_out"], e_r + 1e-30, "r_out")
    e_rh, rel2 = hat_error(F["r_out"], e_r, F["rh"], st[:, 2:3], st[:, 3:4])
    near(h, F["h"], (np.abs(v["g2"]) * e_rh + 4 * U * (np.abs(F["rh"] * v["g2"]) + np.abs(v["b2"]))) * (1 + BF) + BF * np.abs(F["h"]) + 1e-30, "h")
    size1, size2 = np.abs(n["y"]).mean(1, keepdims=True), np.abs(F["r_out"]).mean(1, keepdims=True)
    tol = np.concatenate([S * size1, st[:, 1:2] * rel1 * 2, S * size2 + e_r.mean(1, keepdims=True), st[:, 3:4] * rel2 * 2], 1)
    near(stats, st, tol + 1e-30, "stats")
    # backward from the saved values that the forward pass gave
    R, tol = backward(c, n["y"], r_out.double().cpu().numpy(), stats.double().cpu().numpy(), n["dh"], n["dr"], v, gate, groups)
    got = dict(zip(("dy", "dr", "dg1", "db1", "dg2", "db2", "dgate"), call_bwd(c, t, r_out, stats, gate_rows)))
    assert (got["db1"] is None) == (not shift) and (got["db2"] is None) == (not shift) and (got["dgate"] is None) == (gate_rows is None)
    for name, g in got.items():
        if g is not None:
            near(g, R[name], tol[name], name)
    # no gradient through the residual stream: the same as zeros
    a = call_bwd(c, dict(t, dr=None), r_out, stats, gate_rows)
    b = call_bwd(c, dict(t, dr=torch.zeros_like(t["r"])), r_out, stats, gate_rows)
    assert all(x is y or torch.equal(x, y) for x, y in zip(a, b))


@gpu
def test_rows_far_from_zero():
    """A mean a thousand times the deviation: the variance is not formed from the squares alone."""
    for kind in ("layer", "rms"):
        c, t, n, v, gate, _ = make(64, 512, kind, True, 64, mean=1000.0)
        F = forward(c, n["y"], n["r"], v, gate)
        r_out, h, stats = call_fwd(c, t, 64)
        st = F["stats"]
        e_yh, _ = hat_error(n["y"], np.zeros_like(n["y"]), F["yh"], st[:, 0:1], st[:, 1:2])
        e_n = np.abs(v["g1"]) * e_yh + 4 * U * (np.abs(F["yh"] * v["g1"]) + np.abs(v["b1"]))
        near(r_out, F["r_out"], np.abs(gate) * e_n + 4 * U * (np.abs(gate * F["n"]) + np.abs(gate * v["b1"]) + np.abs(c["scale"] * n["r"])), "r_out")


@gpu
def test_rows_without_spread_and_rows_with_nan():
    """Constant rows: their deviation is sqrt(eps).  A row of NaN leaves the other rows as they are."""
    import torch
    for d in (16, 64, 1032):
        c, t, n, v, gate, _ = make(50, d, "layer", True, 50)
        t["y"][7] = 3.0
        t["y"][8] = 0.0
        clean = call_fwd(c, t, 50)
        assert torch.isfinite(clean[1].float()).all() and abs(float(clean[2][8, 1]) * math.sqrt(c["eps"]) - 1) < 1e-6
        t["y"][20] = float("nan")
        t["r"][21, 3] = float("inf")
        got = call_fwd(c, t, 50)
        keep = [i for i in range(50) if i not in (20, 21)]
        for a, b in zip(clean, got):
            assert torch.equal(a[keep], b[keep])
        assert torch.isnan(got[1][20].float()).all()
        a = call_bwd(c, dict(t, gate=None), clean[0], clean[2], 0)
        assert torch.isnan(a[0][20].float()).all() and torch.isfinite(a[0][keep].float()).all()


@gpu
def test_in_place_residual_and_gradient():
    import torch
    from paper_2509_22418_b200 import ppu
    for T, d, rows in ((1000, 264, 1000), (2000, 64, 1), (130, 2048, 130)):
        c, t, *_ = make(T, d, "layer", True, rows)
        r_out, h, stats = call_fwd(c, t, rows)
        t2 = dict(t, r=t["r"].clone())
        r2, h2, s2 = call_fwd(c, t2, rows, in_place=True)
        assert r2.data_ptr() == t2["r"].data_ptr() and torch.equal(r2, r_out) and torch.equal(h2, h) and torch.equal(s2, stats)
        ref = call_bwd(c, t, r_out, stats, rows)
        dr = t["dr"].clone()
        o = [torch.empty_like(x) for x in ref]
        n = C.c_size_t()
        assert ppu.lib().ppu_norm_gate_query_bytes(T, d, rows, C.byref(n)) == 0
        ws = torch.full((n.value + 256,), 0xA5, dtype=torch.uint8, device="cuda")
        p = lambda x: C.c_void_p(x.data_ptr())  # noqa: E731
        rc = ppu.lib().ppu_norm_gate_bwd(p(t["dh"]), p(dr), p(t["y"]), p(r_out), p(stats), p(t["gate"]), rows, p(t["g1"]), p(t["b1"]), p(t["g2"]), 0,
                                         C.c_float(c["scale"]), p(o[0]), p(dr), p(o[2]), p(o[3]), p(o[4]), p(o[5]), p(o[6]), T, d, p(ws), n,
                                         C.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert rc == 0
        torch.cuda.synchronize()
        o[1] = dr
        assert all(torch.equal(a, b) for a, b in zip(o, ref)) and bool((ws[n.value:] == 0xA5).all())


@gpu
def test_surroundings_are_untouched():
    import torch
    from paper_2509_22418_b200 import ppu
    p = lambda x: C.c_void_p(x.data_ptr())  # noqa: E731
    for T, d in ((5, 8), (77, 264), (3, 4096)):
        c, t, *_ = make(T, d, "layer", True, None)
        ref = call_fwd(c, t, None)
        r = torch.full((T + 2, d), 7.0, device="cuda")
        h = torch.full((T + 2, d), 7.0, dtype=torch.bfloat16, device="cuda")
        s = torch.full((T + 2, 4), 7.0, device="cuda")
        rc = ppu.lib().ppu_norm_gate_fwd(p(t["y"]), p(t["r"]), None, 0, p(t["g1"]), p(t["b1"]), p(t["g2"]), p(t["b2"]), 0, C.c_float(c["scale"]),
                                         C.c_float(c["eps"]), p(r[1:]), p(h[1:]), p(s[1:]), T, d, C.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert rc == 0
        torch.cuda.synchronize()
        for got, want in ((r, ref[0]), (h, ref[1]), (s, ref[2])):
            assert torch.equal(got[1:-1], want) and bool((got[0] == 7).all()) and bool((got[-1] == 7).all())


@gpu
def test_gradients_against_differences():
    """f = sum(h H) + sum(r_out D) of the definition in 64 bits, differentiated numerically."""
    T, d, rows = 12, 40, 4
    for kind in ("layer", "rms"):
        c, t, n, v, gate, groups = make(T, d, kind, True, rows, seed=3)
        r_out, _, stats = call_fwd(c, t, rows)
        got = [g.double().cpu().numpy() for g in call_bwd(c, t, r_out, stats, rows)]

        def f(y, r, g1, b1, g2, b2, gt):
            F = forward(c, y, r, dict(g1=g1, b1=b1, g2=g2, b2=b2), gt[np.arange(T) // rows])
            return (F["h"] * n["dh"]).sum() + (F["r_out"] * n["dr"]).sum()
        args = [n["y"], n["r"], v["g1"], v["b1"], v["g2"], v["b2"], n["gate"]]
        rng = np.random.default_rng(5)
        for i, g in enumerate(got):
            for _ in range(3):
                D = rng.standard_normal(g.shape)
                step = 1e-6
                plus, minus = list(args), list(args)
                plus[i], minus[i] = args[i] + step * D, args[i] - step * D
                diff = (f(*plus) - f(*minus)) / (2 * step)
                # dy is rounded to bf16, the others to fp32
                assert abs(diff - (g * D).sum()) <= (2 * BF if i == 0 else 1e-5) * (np.abs(g) * np.abs(D)).sum() + 1e-8, (kind, i)


@gpu
def test_captured_streamed_and_repeated_calls_have_the_same_bits():
    import torch
    for rows in (1500, 1, 100):
        c, ta, *_ = make(1500, 264, "layer", True, rows, seed=1)
        _, tb, *_ = make(1500, 264, "layer", True, rows, seed=2)

        def both(t):
            out = call_fwd(c, t, rows)
            return out + call_bwd(c, t, out[0], out[2], rows)
        ref_a, ref_b = both(ta), both(tb)
        s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
        s1.wait_stream(torch.cuda.current_stream())
        s2.wait_stream(torch.cuda.current_stream())
        for _ in range(3):
            with torch.cuda.stream(s1):
                got_a = both(ta)
            with torch.cuda.stream(s2):
                got_b = both(tb)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(ref_a + ref_b, got_a + got_b))
        t = {k: x.clone() for k, x in ta.items()}
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = both(t)
        for src, ref in ((tb, ref_b), (ta, ref_a)):
            for k in t:
                t[k].copy_(src[k])
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(out, ref))


@gpu
def test_offsets_beyond_32_bits():
    import torch
    T, d = (1 << 20) + 5, 2064              # 2.2 billion elements a tensor
    c, t, n, v, gate, _ = make(3, d, "rms", False, None)
    y = torch.zeros((T, d), dtype=torch.bfloat16, device="cuda")
    r = torch.zeros((T, d), device="cuda")
    y[-3:], r[-3:] = t["y"], t["r"]
    small = call_fwd(c, t, None)
    r_out, h, stats = call_fwd(c, dict(t, y=y, r=r), None, in_place=True)
    for a, b in zip((r_out, h, stats), small):
        assert torch.equal(a[-3:], b)
    del h
    dh = torch.zeros((T, d), dtype=torch.bfloat16, device="cuda")
    dh[-3:] = t["dh"]
    got = call_bwd(c, dict(t, y=y, dh=dh, dr=None), r_out, stats, None)
    want = call_bwd(c, dict(t, dr=None), small[0], small[2], None)
    assert torch.equal(got[0][-3:], want[0]) and torch.equal(got[1][-3:], want[1]) and not got[0][:-3].any()


@gpu
def test_no_rows():
    import torch
    c, t, *_ = make(4, 64, "layer", True, None)
    z = {k: (x[:0] if k in ("y", "r", "dh", "dr") else x) for k, x in t.items() if x is not None}
    z["gate"] = None
    r_out, h, stats = call_fwd(c, z, None)
    assert r_out.shape == (0, 64) and stats.shape == (0, 4)
    got = call_bwd(c, z, r_out, stats, None)
    assert got[0].shape == (0, 64) and not any(bool(x.any()) for x in got[2:6])
    torch.cuda.synchronize()


# ---- refusals, on the host ----------------------------------------------------------------------
@pytest.fixture(scope="module")
def ppu():
    from paper_2509_22418_b200 import build, ppu as mod
    build.build()
    return mod


def _base():
    buf = (C.c_uint8 * 65536)()
    return buf, (C.addressof(buf) + 255) & ~255


FWD = ["y", "r", "gate", "gate_rows", "g1", "b1", "g2", "b2", "kind", "scale", "eps", "r_out", "h", "stats", "T", "d", "st"]
BWD = ["dh", "dr_out", "y", "r_out", "stats", "gate", "gate_rows", "g1", "b1", "g2", "kind", "scale", "dy", "dr", "dg1", "db1", "dg2", "db2", "dgate", "T", "d",
       "ws", "nb", "st"]


def _call(ppu, names, fn, **change):
    keep, base = _base()
    a = {n: C.c_void_p(base) for n in names}
    a.update(gate=None, gate_rows=0, kind=0, scale=C.c_float(1.0), eps=C.c_float(1e-5), T=4, d=64, st=None, nb=C.c_size_t(1 << 40), dgate=None)
    for n, x in change.items():
        a[n] = C.c_void_p(base + 4) if x == "odd" else C.c_void_p(base) if x == "there" else x
    rc = fn(*[a[n] for n in names])
    del keep
    return rc


@pytest.mark.parametrize("change,code", [
    (dict(y=None), -1), (dict(r=None), -1), (dict(g1=None), -1), (dict(g2=None), -1), (dict(h=None), -1), (dict(r_out=None), -1), (dict(stats=None), -1),
    (dict(d=60), -2), (dict(d=4104), -2), (dict(d=0), -1), (dict(T=-1), -1), (dict(T=(1 << 24) + 1), -2), (dict(kind=2), -1), (dict(eps=C.c_float(-1.0)), -1),
    (dict(eps=C.c_float(math.nan)), -1), (dict(gate="there", gate_rows=0), -1), (dict(gate="there", gate_rows=-3), -1), (dict(y="odd"), -1), (dict(r="odd"), -1),
    (dict(b1="odd"), -1), (dict(stats="odd"), -1), (dict(gate="odd", gate_rows=4), -1),
])
def test_forward_refuses(ppu, change, code):
    assert _call(ppu, FWD, ppu.lib().ppu_norm_gate_fwd, **change) == code


@pytest.mark.parametrize("change,code", [
    (dict(dh=None), -1), (dict(y=None), -1), (dict(r_out=None), -1), (dict(stats=None), -1), (dict(g1=None), -1), (dict(dy=None), -1), (dict(dr=None), -1),
    (dict(dg1=None), -1), (dict(dg2=None), -1), (dict(ws=None), -1), (dict(nb=C.c_size_t(8)), -4), (dict(gate="there", gate_rows=2), -1), (dict(dgate="there"), -1),
    (dict(gate="there", dgate="there", gate_rows=0), -1), (dict(d=20), -2), (dict(kind=-1), -1), (dict(dr_out="odd"), -1), (dict(ws="odd"), -1),
])
def test_backward_refuses(ppu, change, code):
    assert _call(ppu, BWD, ppu.lib().ppu_norm_gate_bwd, **change) == code


def test_workspace_sizes(ppu):
    n = C.c_size_t()
    for T, d, rows in ((1, 8, 0), (8192, 2048, 8192), (8192, 2048, 1), (8192, 2048, 77), (1 << 20, 64, 5), (0, 64, 0)):
        assert ppu.lib().ppu_norm_gate_query_bytes(T, d, rows, C.byref(n)) == 0
        assert n.value <= 5 * 4 * d * min(max(T, 0), 2368 * 2)
    for T, d, rows in ((-1, 8, 0), (1, 12, 0), (1, 8, -1)):
        assert ppu.lib().ppu_norm_gate_query_bytes(T, d, rows, C.byref(n)) < 0
    assert ppu.lib().ppu_norm_gate_query_bytes(1, 8, 0, None) == -1


def test_tensors_are_checked(ppu):
    import torch
    y, r, g, s = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 64), torch.ones(64), torch.zeros(4, 4)
    with pytest.raises(ppu.PpuError):
        ppu.ppu_norm_gate_fwd(y, r, g, g)
    with pytest.raises(ppu.PpuError):
        ppu.ppu_norm_gate_bwd(y, r, y, r, s, g, g)


@gpu
def test_device_tensors_are_checked():
    import torch
    from paper_2509_22418_b200 import ppu
    c = dict(device="cuda")
    y, r, g, s = torch.zeros(4, 64, dtype=torch.bfloat16, **c), torch.zeros(4, 64, **c), torch.ones(64, **c), torch.zeros(4, 4, **c)
    for args in ((y.float(), r, g, g), (y, r.bfloat16(), g, g), (y, r[:3], g, g), (y, r, g[:32], g), (y, r, g, g.double()), (y, r.cpu(), g, g),
                 (y.t(), r.t(), g, g), (torch.zeros(4, 128, dtype=torch.bfloat16, **c)[:, ::2], r, g, g)):
        with pytest.raises(ppu.PpuError):
            ppu.ppu_norm_gate_fwd(*args)
    for kw in (dict(kind="batch"), dict(gate=torch.zeros(4, 64, **c)), dict(gate=torch.zeros(1, 64, **c), gate_rows=2), dict(gate=g, gate_rows=4),
               dict(gate=torch.zeros(4, 64, **c), gate_rows=-1), dict(post_shift=g[:8]), dict(eps=-1.0)):
        with pytest.raises(ppu.PpuError):
            ppu.ppu_norm_gate_fwd(y, r, g, g, **kw)
    for args in ((y.float(), r, y, r, s, g, g), (y, r.half(), y, r, s, g, g), (y, r, y, r, s[:, :2], g, g), (y[:3], r, y, r, s, g, g)):
        with pytest.raises(ppu.PpuError):
            ppu.ppu_norm_gate_bwd(*args)


@gpu
def test_writing_in_place_is_seen_by_autograd():
    """A graph that saved r is told that r has changed; an r of a graph of its own is not overwritten."""
    import torch
    from paper_2509_22418_b200 import ppu
    y, g = torch.randn(4, 64, device="cuda").bfloat16(), torch.ones(64, device="cuda")
    r = torch.randn(4, 64, device="cuda")
    w = torch.ones(64, device="cuda", requires_grad=True)
    loss = (r * w).sum()
    before = r._version
    out = ppu.ppu_norm_gate_fwd(y, r, g, g, in_place=True)
    assert out[0] is r and r._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    for own in (r.clone().requires_grad_(), r.clone().requires_grad_() * 2):
        was = own.detach().clone()
        with pytest.raises(ppu.PpuError):
            ppu.ppu_norm_gate_fwd(y, own, g, g, in_place=True)
        assert torch.equal(own.detach(), was)
        with torch.no_grad():
            got = ppu.ppu_norm_gate_fwd(y, own, g, g, in_place=True)
        assert torch.equal(got[0].detach(), ppu.ppu_norm_gate_fwd(y, was, g, g)[0])
    with torch.inference_mode():
        s = r + 0
    assert ppu.ppu_norm_gate_fwd(y, s, g, g, in_place=True)[0] is s


@gpu
def test_in_place_has_to_be_a_truth_value():
    """One that is neither true nor false is an error before r is written."""
    import torch
    from paper_2509_22418_b200 import ppu
    y, r, g = torch.randn(4, 64, device="cuda").bfloat16(), torch.randn(4, 64, device="cuda"), torch.ones(64, device="cuda")
    was = r.clone()
    with pytest.raises(ValueError):
        ppu.ppu_norm_gate_fwd(y, r, g, g, in_place=np.zeros(2))
    assert torch.equal(r, was)


@gpu
@pytest.mark.parametrize("gate_rows", [0, 5])
def test_no_rows_with_a_gate(gate_rows):
    """One row of the gate for all rows is one row also for none of them; its gradient is a sum over nothing."""
    import torch
    from paper_2509_22418_b200 import ppu
    y, r, s, g = (torch.zeros(0, n, device="cuda") for n in (64, 64, 4, 64))
    g = torch.ones(64, device="cuda")
    for rows in (0, 1) if gate_rows == 0 else (0,):
        gate = torch.full((rows, 64), 3.0, device="cuda")
        r_out, h, stats = ppu.ppu_norm_gate_fwd(y.bfloat16(), r, g, g, gate=gate, gate_rows=gate_rows)
        assert r_out.shape == h.shape == (0, 64)
        got = ppu.ppu_norm_gate_bwd(h, r, y.bfloat16(), r_out, stats, g, g, gate=gate, gate_rows=gate_rows)
        assert got[6].shape == gate.shape and not got[6].any() and not got[2].any() and not got[4].any()
    with pytest.raises(ppu.PpuError):
        ppu.ppu_norm_gate_fwd(y.bfloat16(), r, g, g, gate=torch.ones(2, 64, device="cuda"), gate_rows=gate_rows)


@gpu
@pytest.mark.parametrize("T,d,gate_rows", [(300, 256, 300), (777, 64, 100), (1001, 1032, 1), (1500, 264, 7), (97, 4096, None), (350, 2104, 2 ** 31 - 1)])
def test_whatever_the_workspace_held(T, d, gate_rows):
    """Workspaces of all ones (NaN) and of zeros; a gate row for more rows than there are."""
    import torch
    from paper_2509_22418_b200 import ppu
    c, t, *_ = make(T, d, "layer", True, gate_rows)
    r_out, _, stats = call_fwd(c, t, gate_rows)
    n = ppu.ppu_norm_gate_query_bytes(T, d, gate_rows or 0)
    a, b = (call_bwd(c, t, r_out, stats, gate_rows, workspace=torch.full((n,), fill, dtype=torch.uint8, device="cuda")) for fill in (0, 255))
    assert all(x is y or torch.equal(x, y) for x, y in zip(a, b))


@gpu
@pytest.mark.parametrize("which", ["b1", "b2"])
@pytest.mark.parametrize("gate_rows", [None, 257, 1])
def test_one_shift_alone(which, gate_rows):
    """A shift of zeros in the place of one that is not there: the same bits, and no gradient for it."""
    import torch
    from paper_2509_22418_b200 import ppu
    c, t, *_ = make(257, 264, "layer", True, gate_rows, seed=9)
    some, zeros = dict(t, **{which: None}), dict(t, **{which: torch.zeros(264, device="cuda")})
    a, b = call_fwd(c, some, gate_rows), call_fwd(c, zeros, gate_rows)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    a, b = call_bwd(c, some, a[0], a[2], gate_rows), call_bwd(c, zeros, b[0], b[2], gate_rows)
    left_out = 3 if which == "b1" else 5
    assert a[left_out] is None and b[left_out] is not None
    assert all(torch.equal(x, y) for i, (x, y) in enumerate(zip(a, b)) if i != left_out and y is not None)
