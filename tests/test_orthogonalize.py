"""The orthogonalised update (ppu_orthogonalize) against its definition in 64 bits.

Two references.  `definition` is the formula.  `model` is the same with the kernels' documented roundings and no others: the products' operands in
fp16 (times 2^12) but for P's diagonal, which is kept for shorter sides below 256, and X, which is carried beside the fp16 copy that P multiplies; where the shorter side is at
most 128 and the longer at most 2048 P multiplies a pair of fp16.  How far the model is from the definition is what the arithmetic itself costs; the kernels may be as far, in
root mean square, plus the result's rounding (uniform within half a step of 2^-8: 2^-8 / sqrt(3) of the value at most) and a quarter for the fp32 sums.

Element by element: a sum whose last bits differ puts one in a hundred of the values that are then rounded to fp16 on the other side, and from there on
all roundings are others (the model with its sums changed by 1e-7 is as far from itself as from the definition, and its largest error then is 4.6 to 7.4
times the root mean square).  So the kernels' errors are not the model's but are distributed like them: sums of many roundings, of which those on
the diagonal of P act on a whole row and make its root mean square up to twice the others'; six deviations cover 10^6 values: 12 times the cost, beside
half a step of bf16.  In a matrix of a few values the model may have no error by luck where the kernels round X to fp16 the other way, times a diagonal
of P up to 2.8 against an X' of 0.65 of X: 2^-12 * 2.8 / 0.65 for each of five steps, below 2^-7 of the value."""
import ctypes as C
import math

import numpy as np
import pytest

gpu = pytest.mark.gpu
U, BF = 2.0 ** -24, 2.0 ** -8
COEF = (3.4445, -4.7750, 2.0315)


def f32(x):
    return float(np.float32(x))


def triples(coef, steps):
    return [tuple(f32(x) for x in (coef[k] if hasattr(coef[0], "__len__") else coef)) for k in range(steps)]


def start(u, eps):
    return u / (np.sqrt((u * u).sum((1, 2), keepdims=True)) + f32(eps))


def definition(u, steps=5, coef=COEF, eps=1e-7, scale=1.0):
    X = start(u, eps)
    for a, b, c in triples(coef, steps):
        if u.shape[1] <= u.shape[2]:
            G = X @ X.transpose(0, 2, 1)
            X = a * X + (b * G + c * G @ G) @ X
        else:
            G = X.transpose(0, 2, 1) @ X
            X = a * X + X @ (b * G + c * G @ G)
    return f32(scale) * X


def h(x, exp=12):
    with np.errstate(over="ignore"):
        return np.ldexp(np.ldexp(x, exp).astype(np.float16).astype(np.float64), -exp)


def off_diagonal(P):
    """P without its diagonal, and the diagonal."""
    k = np.arange(P.shape[1])
    d = P[:, k, k].copy()
    P = P.copy()
    P[:, k, k] = 0.0
    return h(P), d


def model(u, steps=5, coef=COEF, eps=1e-7, scale=1.0):
    X = start(u, eps).astype(np.float32).astype(np.float64)
    for a, b, c in triples(coef, steps):
        hi, left = h(X), u.shape[1] <= u.shape[2]
        G = h(hi @ hi.transpose(0, 2, 1)) if left else h(hi.transpose(0, 2, 1) @ hi)
        P, d = off_diagonal(b * G + c * G @ G) if min(u.shape[1:]) < 256 else (h(b * G + c * G @ G), np.zeros(G.shape[:2]))
        Z = hi + h(X - hi) if min(u.shape[1:]) <= 128 and max(u.shape[1:]) <= 2048 else hi
        X = a * X + d[:, :, None] * Z + P @ Z if left else a * X + d[:, None, :] * Z + Z @ P
    return f32(scale) * X


def rms(x):
    return np.sqrt((x * x).mean((1, 2), keepdims=True))


def matrices(batch, m, n, kind="random", seed=0):
    rng = np.random.default_rng(seed + 1000 * m + n)
    x = rng.standard_normal((batch, m, n))
    if kind == "large directions":
        r = max(1, min(m, n) // 8)
        x = 0.05 * x + rng.standard_normal((batch, m, r)) @ rng.standard_normal((batch, r, n))
    elif kind == "falling":
        q, s, p = np.linalg.svd(x, full_matrices=False)
        x = q * (1.0 / np.arange(1, min(m, n) + 1) ** 2) @ p
    elif kind == "rank one":
        x = rng.standard_normal((batch, m, 1)) * rng.standard_normal((batch, 1, n))
    return x.astype(np.float32)


def near(O, u, **kw):
    got = O.detach().double().cpu().numpy()
    want, mod = definition(u, **kw), model(u, **kw)
    size = rms(want) + 1e-300
    assert np.isfinite(got).all() and got.shape == want.shape
    cost = rms(mod - want) / size
    off = rms(got - want) / size
    assert np.all(off <= 1.25 * cost + BF / math.sqrt(3)), (float(off.max()), float(cost.max()))
    err = np.abs(got - want)
    assert np.all(err <= (BF + 2.0 ** -7) * np.abs(want) + 12 * cost * size), float((err / size).max())
    return float(off.max()), float(cost.max())


def cuda(x, dtype="fp32"):
    import torch
    t = torch.from_numpy(x).cuda()
    return t.bfloat16() if dtype == "bf16" else t


SHAPES = [(1, 1, 1), (2, 1, 5), (2, 7, 1), (3, 8, 8), (1, 33, 100), (2, 100, 33), (5, 64, 72), (1, 128, 128), (2, 129, 130), (1, 203, 333), (1, 333, 203), (3, 256, 640),
          (2, 640, 256), (1, 384, 384), (1, 520, 700), (7, 40, 24), (1, 17, 3000), (1, 2100, 12)]


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("batch,m,n", SHAPES)
def test_against_the_definition(batch, m, n, dtype):
    import torch
    from paper_2509_22418_b200 import ppu
    G = cuda(matrices(batch, m, n), dtype)
    O, new = ppu.ppu_orthogonalize(G)
    assert new is None and O.dtype == torch.bfloat16 and O.is_contiguous()
    near(O, G.double().cpu().numpy())
    if batch == 1:
        assert torch.equal(ppu.ppu_orthogonalize(G[0])[0], O[0])


@gpu
@pytest.mark.parametrize("kind", ["large directions", "falling", "rank one"])
@pytest.mark.parametrize("m,n", [(256, 256), (130, 500), (500, 130), (64, 72)])
def test_matrices_of_unequal_directions(m, n, kind):
    """The small directions are multiplied by hundreds: what is rounded must not grow with them."""
    from paper_2509_22418_b200 import ppu
    x = matrices(2, m, n, kind)
    off, cost = near(ppu.ppu_orthogonalize(cuda(x))[0], x.astype(np.float64))
    assert off <= 5e-3


@gpu
def test_singular_values():
    """Those above 0.003 of the norm come to between 0.65 and 1.25."""
    from paper_2509_22418_b200 import ppu
    O = ppu.ppu_orthogonalize(cuda(matrices(1, 200, 300)))[0][0].double().cpu().numpy()
    s = np.linalg.svd(O, compute_uv=False)
    assert s.min() > 0.65 and s.max() < 1.25


@gpu
@pytest.mark.parametrize("steps,coef", [(0, COEF), (1, COEF), (2, COEF), (12, (2.0, -1.5, 0.5)), (3, [(3.0, -3.0, 1.0), (1.5, -0.5, 0.0), (1.875, -1.25, 0.375)]), (4, (1.5, -0.5, 0.0)),
                                        (1, (1.0, 0.0, 0.0)), (2, (0.0, 0.0, 0.0))])
def test_steps_and_coefficients(steps, coef):
    from paper_2509_22418_b200 import ppu
    for m, n in ((72, 136), (136, 75)):
        x = matrices(2, m, n)
        O, _ = ppu.ppu_orthogonalize(cuda(x), steps=steps, coef=coef, scale=0.2, eps=1e-3)
        near(O, x.astype(np.float64), steps=steps, coef=coef, scale=0.2, eps=1e-3)


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("m,n", [(64, 128), (77, 35)])
def test_momentum(m, n, nesterov, dtype):
    import torch
    from paper_2509_22418_b200 import ppu
    G, old = cuda(matrices(3, m, n), dtype), cuda(matrices(3, m, n, seed=5) * 7)
    was = old.clone()
    beta, weight = 0.9, 0.3
    O, new = ppu.ppu_orthogonalize(G, momentum=old, beta=beta, weight=weight, nesterov=nesterov)
    assert torch.equal(old, was) and new.dtype == torch.float32
    g, p = G.double().cpu().numpy(), old.double().cpu().numpy()
    want = f32(beta) * p + f32(weight) * g
    size = np.abs(f32(beta) * p) + np.abs(f32(weight) * g)
    assert np.all(np.abs(new.double().cpu().numpy() - want) <= 2 * U * size)
    k = new.double().cpu().numpy()
    near(O, f32(weight) * g + f32(beta) * k if nesterov else k)
    O2, new2 = ppu.ppu_orthogonalize(G, momentum=old, beta=beta, weight=weight, nesterov=nesterov, in_place=True)
    assert new2 is old and torch.equal(old, new) and torch.equal(O2, O)


@gpu
def test_a_matrix_of_every_layer_of_a_parameter_vector():
    """Strided rows and matrices are read where they lie; what is between them is not touched."""
    import torch
    from paper_2509_22418_b200 import ppu
    L, m, n = 4, 40, 56
    g = torch.randn(L, 9000, device="cuda")
    mom = torch.randn(L, 7000, device="cuda")
    view = torch.as_strided(g, (L, m, n), (9000, 64, 1), 100)          # rows of 64, of which 56
    mv = torch.as_strided(mom, (L, m, n), (7000, n, 1), 12)
    was = mom.clone()
    want, wm = ppu.ppu_orthogonalize(view.contiguous(), momentum=mv.contiguous())
    O, new = ppu.ppu_orthogonalize(view, momentum=mv)
    assert torch.equal(O, want) and torch.equal(new, wm) and torch.equal(mom, was)
    O, new = ppu.ppu_orthogonalize(view, momentum=mv, in_place=True)
    assert torch.equal(O, want) and torch.equal(mv, wm)
    mv.copy_(torch.as_strided(was, (L, m, n), (7000, n, 1), 12))
    assert torch.equal(mom, was)
    odd = torch.as_strided(g, (L, m, 55), (8999, 61, 1), 3)            # nothing aligned
    assert torch.equal(ppu.ppu_orthogonalize(odd)[0], ppu.ppu_orthogonalize(odd.contiguous())[0])


@gpu
def test_sizes_of_numbers():
    """Matrices as large and as small as fp32 holds, of zeros, with a value that is not finite: each by itself."""
    import torch
    from paper_2509_22418_b200 import ppu
    x = matrices(1, 48, 80)[0]
    big = np.stack([x, x * np.float32(1e37), x * np.float32(1e-30), 0 * x, x])
    G = cuda(big)
    ref = ppu.ppu_orthogonalize(G, eps=0.0)[0]
    near(ref[:3], big[:3].astype(np.float64), eps=0.0)
    assert not ref[3].any() and torch.equal(ref[0], ref[4])
    assert not ppu.ppu_orthogonalize(G)[0][3].any()
    for bad in (float("nan"), float("inf"), -float("inf")):
        G[0, 5, 6] = bad
        got = ppu.ppu_orthogonalize(G, eps=0.0)[0]
        assert torch.isnan(got[0].float()).all() and torch.equal(got[1:], ref[1:])
    small = ppu.ppu_orthogonalize(cuda(big[:1] * np.float32(1e-9)), eps=1e-7)[0]      # the norm is of eps's size
    near(small, (big[:1] * np.float32(1e-9)).astype(np.float64), eps=1e-7)


@gpu
def test_a_single_large_value():
    """X's largest entry is one: no overflow in fp16."""
    from paper_2509_22418_b200 import ppu
    x = np.zeros((1, 100, 200), dtype=np.float32)
    x[0, 3, 7] = -5.0
    near(ppu.ppu_orthogonalize(cuda(x))[0], x.astype(np.float64))
    x[0, np.arange(100), np.arange(100)] = 1.0
    near(ppu.ppu_orthogonalize(cuda(x))[0], x.astype(np.float64))


@gpu
@pytest.mark.parametrize("batch,m,n", [(1, 203, 333), (5, 130, 70)])
def test_captured_streamed_and_repeated_calls_have_the_same_bits(batch, m, n):
    import torch
    from paper_2509_22418_b200 import ppu
    G, old = cuda(matrices(batch, m, n)), cuda(matrices(batch, m, n, seed=3))
    flags = torch.zeros(8, dtype=torch.int32, device="cuda")
    ref = ppu.ppu_orthogonalize(G, momentum=old, flags=flags)
    ppu.ppu_op_status(flags)
    nb = ppu.ppu_orthogonalize_query_bytes(batch, m, n)
    for fill in (0, 255):
        got = ppu.ppu_orthogonalize(G, momentum=old, workspace=torch.full((nb,), fill, dtype=torch.uint8, device="cuda"))
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = ppu.ppu_orthogonalize(G, momentum=old)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        graph.replay()
        with torch.cuda.stream(side):
            other = ppu.ppu_orthogonalize(G, momentum=old)
        torch.cuda.synchronize()
        assert torch.equal(cap[0], ref[0]) and torch.equal(other[0], ref[0])


@gpu
def test_empty():
    import torch
    from paper_2509_22418_b200 import ppu
    for shape in ((0, 4, 8), (3, 0, 8), (3, 4, 0), (0, 8)):
        G = torch.zeros(shape, device="cuda")
        O, new = ppu.ppu_orthogonalize(G, momentum=G)
        assert O.shape == new.shape == shape


@gpu
def test_writing_in_place_is_seen_by_autograd():
    import torch
    from paper_2509_22418_b200 import ppu
    G, mom = torch.randn(16, 24, device="cuda"), torch.randn(16, 24, device="cuda")
    before = mom._version
    ppu.ppu_orthogonalize(G, momentum=mom, in_place=True)
    assert mom._version > before
    leaf = mom.clone().requires_grad_()
    with pytest.raises(ppu.PpuError):
        ppu.ppu_orthogonalize(G, momentum=leaf, in_place=True)


# ---- refusals ----------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def ppu():
    from paper_2509_22418_b200 import build, ppu as mod
    build.build()
    return mod


N = ["G", "ldg", "sg", "gt", "mom", "ldm", "sm", "out", "ldo", "so", "beta", "w", "nest", "coef", "nc", "steps", "eps", "scale", "O", "batch", "m", "n", "ws", "nb", "flags", "st"]


def _call(ppu, **change):
    buf = (C.c_uint8 * 65536)()
    base = (C.addressof(buf) + 255) & ~255
    a = {k: C.c_void_p(base) for k in N}
    a.update({k: C.c_int64(16) for k in ("ldg", "ldm", "ldo")}, **{k: C.c_int64(128) for k in ("sg", "sm", "so")}, gt=1, mom=None, out=None, beta=C.c_float(0.9), w=C.c_float(1),
             nest=1, coef=(C.c_float * 96)(*(COEF * 32)), nc=1, steps=5, eps=C.c_float(1e-7), scale=C.c_float(1), batch=2, m=8, n=16, nb=C.c_size_t(1 << 40), flags=None, st=None)
    for k, x in change.items():
        a[k] = C.c_void_p(base + 2) if x == "odd" else C.c_void_p(base) if x == "there" else C.c_void_p(base + 4096) if x == "else" else x
    return ppu.lib().ppu_orthogonalize(*[a[k] for k in N])


def _coef(*v):
    return (C.c_float * 96)(*(v * 32))


@pytest.mark.parametrize("change,code", [
    (dict(G=None), -1), (dict(O=None), -1), (dict(ws=None), -1), (dict(coef=None), -1), (dict(nb=C.c_size_t(100)), -4), (dict(batch=-1), -1), (dict(batch=65536), -2),
    (dict(m=-1), -1), (dict(m=65537), -2), (dict(n=65537), -2), (dict(batch=65535, m=65536, n=65536), -2), (dict(steps=-1), -1), (dict(steps=33), -1), (dict(nc=2), -1), (dict(nc=0), -1),
    (dict(gt=2), -1), (dict(eps=C.c_float(-1)), -1), (dict(eps=C.c_float(math.nan)), -1), (dict(mom="there"), -1), (dict(out="there"), -1), (dict(ldg=C.c_int64(15)), -1),
    (dict(mom="there", out="else", ldm=C.c_int64(8)), -1), (dict(mom="there", out="else", ldo=C.c_int64(8)), -1), (dict(mom="there", out="else", so=C.c_int64(64)), -1),
    (dict(mom="there", out="there", ldm=C.c_int64(20)), -1), (dict(mom="there", out="there", sm=C.c_int64(130)), -1), (dict(sg=C.c_int64(-4)), -1), (dict(G="odd"), -1),
    (dict(mom="odd", out="there"), -1), (dict(mom="else", out="there"), -1), (dict(O="odd"), -1), (dict(ws="odd"), -1),
    (dict(coef=_coef(4.0, -4.0, 3.0)), -1), (dict(coef=_coef(math.nan, 0.0, 0.0)), -1), (dict(coef=_coef(math.inf, 0.0, 0.0)), -1), (dict(coef=_coef(1.0, 1e30, -1e30)), -1),
    (dict(coef=_coef(-3.0, 0.0, 0.0)), -1), (dict(coef=_coef(3.4445, -4.775, math.nan)), -1),
])
def test_refuses(ppu, change, code):
    assert _call(ppu, **change) == code


def test_workspace_sizes(ppu):
    assert ppu.ppu_orthogonalize_query_bytes(0, 8, 8) == ppu.ppu_orthogonalize_query_bytes(2, 0, 8) == 0
    assert 6 * 8192 * 2048 + 4 * 2048 ** 2 <= ppu.ppu_orthogonalize_query_bytes(1, 8192, 2048) <= 6 * 8192 * 2048 + 64 * 2048 ** 2
    for bad in ((-1, 8, 8, 5), (1, -1, 8, 5), (1, 8, 8, 40), (1, 1 << 33, 8, 5)):
        with pytest.raises(ppu.PpuError):
            ppu.ppu_orthogonalize_query_bytes(*bad)


def test_tensors_are_checked(ppu):
    import torch
    with pytest.raises(ppu.PpuError):
        ppu.ppu_orthogonalize(torch.zeros(8, 8))


@gpu
def test_device_tensors_are_checked():
    import torch
    from paper_2509_22418_b200 import ppu
    G = torch.zeros(2, 8, 16, device="cuda")
    for kw in (dict(momentum=G[:1]), dict(momentum=G.bfloat16()), dict(momentum=G.cpu()), dict(in_place=True), dict(steps=2, coef=[COEF] * 3), dict(coef=(1.0, 2.0)),
               dict(coef=[COEF] * 33, steps=33), dict(coef=(5.0, 0.0, 0.0)), dict(eps=-1.0), dict(workspace=torch.zeros(64, dtype=torch.uint8, device="cuda")),
               dict(momentum=G[:1].expand(2, 8, 16), in_place=True), dict(flags=torch.zeros(8, device="cuda"))):
        with pytest.raises(ppu.PpuError):
            ppu.ppu_orthogonalize(G, **kw)
    for bad in (G.half(), G[0, 0], G.transpose(1, 2), G[None]):
        with pytest.raises(ppu.PpuError):
            ppu.ppu_orthogonalize(bad)


# ---- matrices of many tiles, in 64 bits on the GPU ---------------------------------------------------
def on_gpu(u, rounded, steps=5):
    """The definition (rounded False) or the model of u [batch, m, n]."""
    import torch
    def h(x):
        return (x * 4096).half().double() / 4096 if rounded else x
    left, small = u.shape[1] <= u.shape[2], min(u.shape[1:]) < 256
    X = u / (u.square().sum((1, 2), keepdim=True).sqrt() + f32(1e-7))
    for a, b, c in triples(COEF, steps):
        hi = h(X)
        G = h(hi @ hi.mT if left else hi.mT @ hi)
        P = b * G + c * G @ G
        d = torch.diagonal(P, dim1=1, dim2=2).clone() if small else torch.zeros_like(P[:, 0])
        P = h(P - torch.diag_embed(d))
        X = a * X + (d[:, :, None] * hi + P @ hi if left else d[:, None, :] * hi + hi @ P)
    return X


@gpu
@pytest.mark.parametrize("batch,m,n,momentum", [
    (1, 1536, 1600, False), (1, 1701, 1404, True),       # one matrix, on either side
    (9, 300, 520, True), (9, 520, 301, False), (12, 150, 700, False), (40, 200, 190, True),      # batches, without and with P's diagonal apart
    (1, 2560, 2304, False), (1, 2304, 2567, False),      # a last wave of halves
    (1, 520, 8200, False), (1, 8200, 520, True), (3, 333, 8193, False),      # A in slices of its sums
    (2, 17, 4100, False), (1, 128, 2056, False), (1, 2049, 100, True),       # sides up to 128 that are too long for the chip
    (40, 200, 1281, True), (40, 1281, 190, False), (101, 509, 481, False), (96, 400, 1009, True),      # SM pairs: waves of tiles
    (1, 2048, 8200, False), (1, 8197, 1500, True), (2, 1793, 2047, False),      # SM pairs: large products, A in slices of its sums
])
def test_matrices_of_many_tiles(batch, m, n, momentum):
    import torch
    from paper_2509_22418_b200 import ppu
    g = torch.Generator(device="cuda").manual_seed(m)
    G = torch.randn(batch, m, n, generator=g, device="cuda")
    old = torch.randn(batch, m, n, generator=g, device="cuda") if momentum else None
    flags = torch.zeros(8, dtype=torch.int32, device="cuda")
    O, new = ppu.ppu_orthogonalize(G, momentum=old, flags=flags)
    ppu.ppu_op_status(flags)
    u = G.double() if old is None else G.double() + f32(0.95) * new.double()
    if old is not None:
        assert float((new.double() - (f32(0.95) * old.double() + G.double())).abs().max()) <= 2.0 ** -22 * float(new.abs().max())
    want, mod = on_gpu(u, False), on_gpu(u, True)
    size = want.square().mean((1, 2), keepdim=True).sqrt()
    cost = (mod - want).square().mean((1, 2), keepdim=True).sqrt() / size
    err = (O.double() - want).abs()
    off = err.square().mean((1, 2), keepdim=True).sqrt() / size
    assert bool((off <= 1.25 * cost + BF / math.sqrt(3)).all()), (float(off.max()), float(cost.max()))
    # (up to 7e6 values: seven deviations where near() has six)
    assert bool((err <= (BF + 2.0 ** -7) * want.abs() + 14 * cost * size).all()), float((err / size).max())
    again = ppu.ppu_orthogonalize(G, momentum=old)
    assert torch.equal(again[0], O)
