"""Further calls of the orthogonalised update (ppu_orthogonalize), by the way that their matrices take through the kernels: on chip (sides up to 128, a
cluster to a matrix), or step by step through memory on single SMs or SM pairs.  References and bounds are those of test_orthogonalize.py."""
import math

import numpy as np
import pytest

from test_orthogonalize import BF, COEF, cuda, definition, f32, h, matrices, model, near, off_diagonal, on_gpu, rms, start, triples

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("batch,m,n", [(24, 100, 701), (7, 33, 1999), (3, 2048, 128)])
def test_on_chip_beside_other_work(batch, m, n):
    """Clusters that share the SMs with other streams' kernels, so that their warps' lanes leave waits at different times: the bits stay."""
    import torch
    from paper_2509_22418_b200 import ppu
    x = matrices(batch, m, n)
    G = cuda(x)
    ref = ppu.ppu_orthogonalize(G)[0]
    near(ref, x.astype("float64"))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    a = torch.randn(1024, 1024, device="cuda").bfloat16()
    other = torch.randn(1, 203, 333, device="cuda")
    torch.cuda.synchronize()
    got = []
    for _ in range(6):
        with torch.cuda.stream(streams[0]):
            a @ a
            ppu.ppu_orthogonalize(other)
        for s in streams[1:]:
            with torch.cuda.stream(s):
                got.append(ppu.ppu_orthogonalize(G)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(g, ref) for g in got)


@gpu
@pytest.mark.parametrize("batch,m,n", [(3, 333, 8193), (2, 520, 4100), (2, 8200, 300)])
def test_slices_of_several_matrices(batch, m, n):
    """A in slices of its sums, several matrices at once: their sums lie apart, whatever the workspace held, however often."""
    import torch
    from paper_2509_22418_b200 import ppu
    x = matrices(batch, m, n, "large directions")
    G = cuda(x)
    ref = ppu.ppu_orthogonalize(G)[0]
    near(ref, x.astype("float64"))
    nb = ppu.ppu_orthogonalize_query_bytes(batch, m, n)
    ws = torch.full((nb,), 255, dtype=torch.uint8, device="cuda")
    for _ in range(8):
        assert torch.equal(ppu.ppu_orthogonalize(G, workspace=ws)[0], ref)


@gpu
@pytest.mark.parametrize("momentum", [False, True])
@pytest.mark.parametrize("steps", [0, 1, 5])
@pytest.mark.parametrize("m,n", [(48, 80), (130, 200), (200, 131), (40, 2100)])
def test_values_that_are_not_finite(m, n, steps, momentum):
    """A matrix with one is NaN throughout, without a step too; the others of its batch are as without it."""
    import torch
    from paper_2509_22418_b200 import ppu
    G = cuda(matrices(3, m, n))
    kw = dict(steps=steps, momentum=0.5 * G if momentum else None)
    ref = ppu.ppu_orthogonalize(G, **kw)[0]
    for bad in (float("inf"), -float("inf"), float("nan")):
        for where in ("G", "momentum") if momentum else ("G",):
            g, old = G.clone(), kw["momentum"].clone() if momentum else None
            (g if where == "G" else old)[1, m - 1, 3] = bad
            got = ppu.ppu_orthogonalize(g, **dict(kw, momentum=old))[0]
            assert torch.isnan(got[1]).all() and torch.equal(got[0], ref[0]) and torch.equal(got[2], ref[2])
    assert not ppu.ppu_orthogonalize(0 * G, steps=steps)[0].any() and not ppu.ppu_orthogonalize(G, steps=steps, eps=float("inf"))[0].any()


@gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("m,heads,n", [(96, 5, 40), (300, 4, 136), (70, 3, 33)])
def test_matrices_whose_rows_lie_beside_one_another(m, heads, n, dtype):
    """The heads of one projection W [m, heads n]: a batch of [m, n], read and (the momentum) written where it lies."""
    import torch
    from paper_2509_22418_b200 import ppu
    G, mom = cuda(matrices(1, m, heads * n)[0], dtype), cuda(matrices(1, m, heads * n + 8, seed=1)[0])
    view, mv = G.view(m, heads, n).transpose(0, 1), mom[:, : heads * n].unflatten(1, (heads, n)).transpose(0, 1)
    was = mom.clone()
    want, wm = ppu.ppu_orthogonalize(view.contiguous(), momentum=mv.contiguous())
    O, new = ppu.ppu_orthogonalize(view, momentum=mv)
    assert torch.equal(O, want) and torch.equal(new, wm) and torch.equal(mom, was)
    O, new = ppu.ppu_orthogonalize(view, momentum=mv, in_place=True)
    assert torch.equal(O, want) and torch.equal(mv, wm) and torch.equal(mom[:, heads * n:], was[:, heads * n:])
    for k in (n - 1, 0):                    # rows that overlap in part, or as a whole
        with pytest.raises(ppu.PpuError):
            ppu.ppu_orthogonalize(torch.as_strided(G, (heads, m, n), (k, heads * n, 1)))


@pytest.mark.parametrize("stride,ld,ok", [(16, 32, True), (128, 16, True), (24, 40, True), (15, 32, False), (16, 31, False), (64, 16, False), (0, 32, False)])
def test_momentum_written_must_not_overlap(stride, ld, ok):
    """2 x 8 x 16: accepted strides come as far as the next check (no workspace)."""
    import ctypes as C
    import test_orthogonalize as t
    from paper_2509_22418_b200 import build, ppu
    build.build()
    assert t._call(ppu, mom="there", out="else", so=C.c_int64(stride), ldo=C.c_int64(ld), nb=C.c_size_t(100)) == (-4 if ok else -1)


def against_64_bits(G, old=None):
    """G [batch, m, n] (and a momentum) by ppu_orthogonalize, within the bounds of test_matrices_of_many_tiles; and the same bits again."""
    import torch
    from paper_2509_22418_b200 import ppu
    flags = torch.zeros(8, dtype=torch.int32, device="cuda")
    O, new = ppu.ppu_orthogonalize(G, momentum=old, flags=flags)
    ppu.ppu_op_status(flags)
    u = G.double() if old is None else G.double() + f32(0.95) * new.double()
    off, err, limit, most = distances(O.double(), u)
    assert bool((off <= limit).all()), (float(off.max()), float(limit.min()))
    assert bool((err <= most).all())
    assert torch.equal(ppu.ppu_orthogonalize(G, momentum=old)[0], O)


def distances(O, u):
    """Root mean square of O - O in 64 bits, over its size; each value's; and the bounds of both."""
    want, mod = on_gpu(u, False), on_gpu(u, True)
    size = want.square().mean((1, 2), keepdim=True).sqrt()
    cost = (mod - want).square().mean((1, 2), keepdim=True).sqrt() / size
    err = (O - want).abs()
    return err.square().mean((1, 2), keepdim=True).sqrt() / size, err, 1.25 * cost + BF / math.sqrt(3), (BF + 2.0 ** -7) * want.abs() + 14 * cost * size


@gpu
@pytest.mark.parametrize("batch,m,n", [(32, 384, 2048), (8, 900, 1200), (7, 1024, 1030), (6, 1024, 1024), (24, 256, 2048), (96, 200, 2400), (13, 2500, 260)])
def test_either_side_of_the_choice_of_tiles(batch, m, n):
    """Products of some 30 GFLOP a step, on tiles that are full or not: single SMs and SM pairs."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(n)
    against_64_bits(torch.randn(batch, m, n, generator=g, device="cuda"))


# ---- X's second number --------------------------------------------------------------------------------
# Random matrices hardly need what X's fp16 copy leaves of it: without it their error stays within the bounds.  Matrices of a few large directions do (their
# small directions are multiplied by hundreds, and the copy's rounding with them), on every way through the kernels.
def large_directions(batch, m, n, seed=0):
    """On the GPU: a product of rank min(m, n) / 8 and a twentieth of noise."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed + 1000 * m + n)
    r = min(m, n) // 8
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    return 0.05 * randn(batch, m, n) + randn(batch, m, r) @ randn(batch, r, n)


@gpu
@pytest.mark.parametrize("batch,m,n,momentum", [
    (12, 100, 701, False), (2, 1999, 128, True),                                  # on chip
    (9, 203, 333, True), (5, 640, 250, False), (12, 768, 768, False), (3, 520, 700, True),      # single SMs, with P's diagonal apart and without
    (3, 333, 8193, False), (2, 200, 4100, True), (1, 8200, 520, False),            # single SMs, A in slices
    (96, 200, 2400, False), (130, 1800, 200, True),                                # SM pairs, with P's diagonal apart
    (8, 900, 1200, True), (7, 1100, 1024, False),                                  # and without
    (1, 2560, 2304, False), (1, 2304, 2567, True),                                 # SM pairs, a last wave of halves
    (1, 2048, 8200, False), (1, 8197, 1500, True),                                 # SM pairs, A in slices
])
def test_matrices_of_a_few_large_directions(batch, m, n, momentum):
    G = large_directions(batch, m, n)
    against_64_bits(G, 0.5 * large_directions(batch, m, n, 7) if momentum else None)


def carried(u, second):
    """The model's steps with X carried as its fp16 copy and `second` of what that leaves, rounded to bf16 in the end."""
    X = start(u, 1e-7)
    for k, (a, b, c) in enumerate(triples(COEF, 5)):
        hi = h(X)
        X = hi + second(h(X - hi))
        left = u.shape[1] <= u.shape[2]
        G = h(hi @ hi.transpose(0, 2, 1)) if left else h(hi.transpose(0, 2, 1) @ hi)
        P, d = off_diagonal(b * G + c * G @ G) if min(u.shape[1:]) < 256 else (h(b * G + c * G @ G), np.zeros(G.shape[:2]))
        X = a * X + d[:, :, None] * hi + P @ hi if left else a * X + d[:, None, :] * hi + hi @ P
    m = np.frexp(X)
    return np.ldexp(np.rint(m[0] * 256) / 256, m[1])


@pytest.mark.parametrize("m,n", [(200, 640), (400, 1009), (701, 404), (300, 520)])
def test_the_bounds_see_x_second_number(m, n):
    """Left out, or read 32 columns (a block) further, it takes the model above the bound of the tests before; as it is, not."""
    u = matrices(1, m, n, "large directions").astype(np.float64)
    want, mod = definition(u), model(u)
    size = rms(want)
    limit = 1.25 * rms(mod - want) / size + BF / math.sqrt(3)
    off = {k: float((rms(carried(u, f) - want) / size).max()) for k, f in (("there", lambda x: x), ("none", np.zeros_like), ("shifted", lambda x: np.roll(x, 32, 2)))}
    assert off["there"] <= float(limit.max()) and off["none"] > 2 * float(limit.max()) and off["shifted"] > 2 * float(limit.max()), (off, float(limit.max()))


# ---- coefficients that make X smaller -------------------------------------------------------------------
HALF = (0.5, 0.0, 0.0)


@gpu
@pytest.mark.parametrize("m,n", [(72, 136), (200, 260)])
@pytest.mark.parametrize("steps,coef", [(9, HALF), (12, [HALF] * 9 + [(3.0, -3.0, 1.0)] * 3), (2, (0.0, 0.0, 0.0))])
def test_coefficients_that_make_x_smaller(steps, coef, m, n):
    from paper_2509_22418_b200 import ppu
    x = matrices(2, m, n)
    near(ppu.ppu_orthogonalize(cuda(x), steps=steps, coef=coef, scale=100.0)[0], x.astype(np.float64), steps=steps, coef=coef, scale=100.0)


@pytest.mark.parametrize("coef,steps,code", [(HALF, 32, -1), (HALF, 11, -1), (HALF, 9, -4), ((1e-4, 0.0, 0.0), 1, -1), ((1e-20, 0.0, 0.0), 1, -1), ((0.0, 0.0, 0.0), 32, -4)])
def test_coefficients_that_leave_x_without_digits_are_refused(coef, steps, code):
    """What was carried of X fell below fp16's range step by step: after 32 halvings the result was zeros.  (-4: accepted, no workspace.)"""
    import ctypes as C
    import test_orthogonalize as t
    from paper_2509_22418_b200 import build, ppu
    build.build()
    assert t._call(ppu, coef=t._coef(*coef), steps=steps, nb=C.c_size_t(100)) == code
