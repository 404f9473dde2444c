"""Embedding lookup with a scale and the table's gradient (ppu_embed_fwd / _bwd) against their definitions in 64 bits, element by element.

Tolerances: u = 2^-24 (fp32, half a step).  The lookup is one product, rounded once more where the result is bf16 (half a step 2^-8).  The
gradient of an id with n tokens is n - 1 additions in some order, a product and an addition: (n + 2) u of the sum of magnitudes, and the
result's own rounding."""
import ctypes as C

import numpy as np
import pytest

gpu = pytest.mark.gpu
U, BF = 2.0 ** -24, 2.0 ** -8


def words(rng, T, V, kind):
    if kind == "uniform":
        ids = rng.integers(0, V, T)
    elif kind == "zipf":
        ids = (np.exp(rng.random(T) * np.log(V + 1.0)).astype(np.int64) - 1) * 7919 % V
    elif kind == "one":
        ids = np.full(T, V // 2)
    else:
        ids = rng.integers(0, V, T)
        ids[rng.random(T) < 0.4] = -1
        if kind == "none":
            ids[:] = -5
    return ids.astype(np.int32)


def make(T, d, V, kind="uniform", dtype="fp32", seed=0):
    import torch
    rng = np.random.default_rng(seed + T + 3 * d + 7 * V)
    t = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    ids = words(rng, T, V, kind)
    dout = torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).to(t)
    return ids, torch.from_numpy(ids).cuda(), dout.cuda(), dout.double().numpy()


def gradient(ids, dout, V, scale=1.0, add=None):
    """dE, its tolerance without the result's rounding."""
    there = (ids >= 0) & (ids < V)
    dE, size, count = np.zeros((V, dout.shape[1])), np.zeros((V, dout.shape[1])), np.zeros(V)
    np.add.at(dE, ids[there], dout[there])
    np.add.at(size, ids[there], np.abs(dout[there]))
    np.add.at(count, ids[there], 1)
    base = np.zeros_like(dE) if add is None else add
    return dE * scale + base, (count[:, None] + 2) * U * (size * abs(scale) + np.abs(base)) + 1e-37


def near(got, want, tol, name=""):
    g = got.detach().double().cpu().numpy()
    if got.element_size() == 2:
        tol = tol * (1 + BF) + BF * np.abs(want)
    assert g.shape == want.shape and np.all(np.abs(g - want) <= tol), (name, float(np.abs(g - want).max()))


FWD = [(1, 8, 1), (1, 2048, 100), (7, 24, 5), (300, 264, 1000), (1000, 768, 33), (33, 16384, 40), (70000, 8, 9)]


@gpu
@pytest.mark.parametrize("table", ["bf16", "fp32"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,d,V", FWD)
def test_lookup_against_the_definition(T, d, V, table, dtype):
    import torch
    from paper_2509_22418_b200 import ppu
    rng = np.random.default_rng(T + d)
    E = torch.from_numpy(rng.standard_normal((V, d)).astype(np.float32)).to({"bf16": torch.bfloat16, "fp32": torch.float32}[table])
    ids = words(rng, T, V, "padded")
    scale = np.float32(27.7)
    out = ppu.ppu_embed_fwd(torch.from_numpy(ids).cuda(), E.cuda(), scale=float(scale), dtype=dtype)
    assert out.dtype == {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    want = np.where(ids[:, None] >= 0, E.double().numpy()[np.maximum(ids, 0)], 0.0) * float(scale)
    near(out, want, U * np.abs(want))


BWD = [
    # T, d, V, ids: one block sorts up to 16384 tokens, 1, 4, 8 or 16 a thread
    (1, 8, 1, "uniform"), (1, 2048, 100, "uniform"), (5, 8, 3, "uniform"), (31, 40, 7, "padded"), (32, 16, 2, "uniform"), (33, 264, 1, "uniform"),
    (300, 776, 50, "zipf"), (1023, 64, 255, "uniform"), (1024, 64, 256, "padded"), (1025, 72, 257, "zipf"), (1000, 264, 20, "one"), (4096, 32, 65535, "zipf"),
    (4097, 8, 65536, "uniform"), (5000, 520, 30, "one"), (8192, 16, 1000, "padded"), (8193, 24, 70000, "zipf"), (16384, 8, 3, "uniform"), (16383, 16, 300, "one"),
    (700, 8, 1 << 22, "uniform"), (64, 16384, 9, "zipf"), (50, 64, 12, "none"),
    # several blocks, one to three passes
    (16385, 8, 100, "uniform"), (20000, 40, 300, "zipf"), (17000, 16, 40000, "padded"), (70000, 8, 5, "one"), (30000, 8, 1 << 22, "zipf"), (33333, 136, 1000, "uniform"),
]


@gpu
@pytest.mark.parametrize("dtype,grad", [("fp32", "bf16"), ("bf16", "fp32"), ("bf16", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("T,d,V,kind", BWD)
def test_gradient_against_the_definition(T, d, V, kind, dtype, grad):
    import torch
    from paper_2509_22418_b200 import ppu
    ids, it, dout, n = make(T, d, V, kind, dtype)
    scale = float(np.float32(0.7))
    want, tol = gradient(ids, n, V, scale)
    near(ppu.ppu_embed_bwd(it, dout, V, scale=scale, dtype=grad), want, tol)
    if V * d > 1 << 24:
        return
    add = torch.randn(V, d, device="cuda").to({"bf16": torch.bfloat16, "fp32": torch.float32}[grad])
    was = add.clone()
    want, tol = gradient(ids, n, V, scale, add.double().cpu().numpy())
    out = ppu.ppu_embed_bwd(it, dout, V, scale=scale, add=add)
    near(out, want, tol, "add")
    assert torch.equal(add, was)
    again = ppu.ppu_embed_bwd(it, dout, V, scale=scale, add=add, in_place=True)
    assert again is add and torch.equal(out, add)


@gpu
def test_many_tokens():
    import torch
    from paper_2509_22418_b200 import ppu
    T, d, V = 1 << 20, 8, 50000
    for kind in ("zipf", "one"):
        ids, it, dout, n = make(T, d, V, kind)
        want, tol = gradient(ids, n, V)
        near(ppu.ppu_embed_bwd(it, dout, V, dtype="fp32"), want, tol, kind)


@gpu
def test_offsets_beyond_32_bits():
    import torch
    from paper_2509_22418_b200 import ppu
    V, d = (1 << 21) + 5, 1040                 # 2.2 billion elements of the table
    E = torch.zeros((V, d), dtype=torch.bfloat16, device="cuda")
    E[-2:] = torch.randn(2, d, device="cuda").bfloat16()
    ids = torch.tensor([V - 1, 3, V - 2], dtype=torch.int32, device="cuda")
    out = ppu.ppu_embed_fwd(ids, E, dtype="bf16")
    assert torch.equal(out[0], E[-1]) and torch.equal(out[2], E[-2]) and not out[1].any()
    g = torch.randn(3, d, device="cuda")
    dE = ppu.ppu_embed_bwd(ids, g, V)
    assert torch.equal(dE[-1], g[0].bfloat16()) and torch.equal(dE[3], g[1].bfloat16()) and torch.equal(dE[-2], g[2].bfloat16()) and not dE[4:-2].any() and not dE[:3].any()
    del E, dE
    T = (1 << 20)                              # and of the gradient's rows
    big = torch.zeros((T, 2056), dtype=torch.bfloat16, device="cuda")
    big[-1] = g[0, 0]
    ids = torch.zeros(T, dtype=torch.int32, device="cuda")
    ids[-1] = 1
    dE = ppu.ppu_embed_bwd(ids, big, 2)
    assert torch.equal(dE[1], big[-1]) and not dE[0].any()
    out = ppu.ppu_embed_fwd(ids, dE, dtype="bf16")
    assert torch.equal(out[-1], dE[1]) and not out[:-1].any()


@gpu
def test_ids_outside_the_table_are_left_out_and_reported():
    import torch
    from paper_2509_22418_b200 import ppu
    for T in (40, 3000, 20000):
        ids, it, dout, n = make(T, 16, 50)
        flags = torch.zeros(8, dtype=torch.int32, device="cuda")
        E = torch.randn(50, 16, device="cuda")
        a = ppu.ppu_embed_fwd(it, E, flags=flags)
        ppu.ppu_embed_bwd(it, dout, 50, flags=flags)
        ppu.ppu_op_status(flags)
        ids[7] = 50
        ids[-1] = 2 ** 31 - 1
        ids[9] = -2 ** 31
        bad = torch.from_numpy(ids).cuda()
        for call in (lambda f: ppu.ppu_embed_fwd(bad, E, flags=f), lambda f: ppu.ppu_embed_bwd(bad, dout, 50, dtype="fp32", flags=f)):
            got = call(flags)
            with pytest.raises(ppu.PpuError) as e:
                ppu.ppu_op_status(flags)
            assert e.value.code == -8
            assert torch.equal(call(None), got)
        keep = [i for i in range(T) if i not in (7, 9, T - 1)]
        out = ppu.ppu_embed_fwd(bad, E)
        assert not out[[7, 9, T - 1]].any() and torch.equal(out[keep], a[keep])
        want, tol = gradient(ids, n, 50)
        near(got, want, tol)


@gpu
def test_rows_of_absent_tokens_may_hold_anything():
    """NaN and infinities where a token is absent are not read into any sum; elsewhere they stay with their id."""
    import torch
    from paper_2509_22418_b200 import ppu
    ids, it, dout, n = make(3000, 72, 200, "padded")
    clean = ppu.ppu_embed_bwd(it, dout, 200)
    dout[it < 0] = float("nan")
    assert torch.equal(ppu.ppu_embed_bwd(it, dout, 200), clean)
    t = int(np.flatnonzero(ids >= 0)[17])
    dout[t] = float("inf")
    got = ppu.ppu_embed_bwd(it, dout, 200)
    others = [v for v in range(200) if v != ids[t]]
    assert torch.isinf(got[ids[t]]).all() and torch.equal(got[others], clean[others])


@gpu
def test_strided_operands_and_untouched_surroundings():
    import torch
    from paper_2509_22418_b200 import ppu
    ids, it, dout, n = make(500, 40, 90, "zipf", "bf16")
    wide = torch.full((500, 64), float("nan"), device="cuda", dtype=torch.bfloat16)
    wide[:, 8:48] = dout
    want = ppu.ppu_embed_bwd(it, dout, 90)
    assert torch.equal(ppu.ppu_embed_bwd(it, wide[:, 8:48], 90), want)
    table = torch.full((92, 56), 3.0, device="cuda", dtype=torch.bfloat16)
    base = torch.randn(90, 40, device="cuda").bfloat16()
    table[1:91, 8:48] = base
    got = ppu.ppu_embed_bwd(it, dout, 90, add=table[1:91, 8:48])
    assert torch.equal(got, ppu.ppu_embed_bwd(it, dout, 90, add=base))
    ppu.ppu_embed_bwd(it, dout, 90, add=table[1:91, 8:48], in_place=True)
    assert torch.equal(table[1:91, 8:48], got)
    table[1:91, 8:48] = 3.0
    assert bool((table == 3.0).all())
    E = torch.full((90, 48), float("nan"), device="cuda")
    E[:, :40] = base.float()
    assert torch.equal(ppu.ppu_embed_fwd(it, E[:, :40]), ppu.ppu_embed_fwd(it, base.float()))
    assert torch.equal(ppu.ppu_embed_fwd(it, E[:, :40])[:, 3], base.float()[it.long(), 3])


@gpu
@pytest.mark.parametrize("T,V", [(257, 100), (5000, 30), (20000, 1000)])
def test_captured_streamed_and_repeated_calls_have_the_same_bits(T, V):
    import torch
    from paper_2509_22418_b200 import ppu
    ids, it, dout, n = make(T, 136, V, "zipf")
    ref = ppu.ppu_embed_bwd(it, dout, V, dtype="fp32")
    nb = ppu.ppu_embed_query_bytes(T, 136, V)
    for fill in (0, 255):                      # whatever the workspace held
        ws = torch.full((nb,), fill, dtype=torch.uint8, device="cuda")
        assert torch.equal(ppu.ppu_embed_bwd(it, dout, V, dtype="fp32", workspace=ws), ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cap = ppu.ppu_embed_bwd(it, dout, V, dtype="fp32")
        out = ppu.ppu_embed_fwd(it, cap)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        graph.replay()
        with torch.cuda.stream(side):
            other = ppu.ppu_embed_bwd(it, dout, V, dtype="fp32")
        torch.cuda.synchronize()
        assert torch.equal(cap, ref) and torch.equal(other, ref) and torch.equal(out, ref[it.long()])


@gpu
def test_no_tokens():
    import torch
    from paper_2509_22418_b200 import ppu
    ids, x = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, 64, device="cuda")
    add = torch.randn(10, 64, device="cuda")
    assert ppu.ppu_embed_fwd(ids, add).shape == (0, 64)
    dE = ppu.ppu_embed_bwd(ids, x, 10)
    assert dE.shape == (10, 64) and not dE.any()
    assert torch.equal(ppu.ppu_embed_bwd(ids, x, 10, add=add), add)
    assert ppu.ppu_embed_bwd(ids, x, 10, add=add, in_place=True) is add


@gpu
def test_gradient_against_differences():
    """A change of the table changes sum(out * dout) by sum(change * dE): the pair is linear, so any step will do."""
    import torch
    from paper_2509_22418_b200 import ppu
    ids, it, dout, n = make(777, 64, 100, "padded")
    E, step = torch.randn(100, 64, device="cuda"), torch.randn(100, 64, device="cuda")
    f = lambda E: float((ppu.ppu_embed_fwd(it, E, scale=2.0).double() * dout.double()).sum())  # noqa: E731
    dE = ppu.ppu_embed_bwd(it, dout, 100, scale=2.0, dtype="fp32")
    size = float((dout.double().abs() * ppu.ppu_embed_fwd(it, E.abs() + step.abs() * 2, scale=2.0).double()).sum())
    assert abs(f(E + step) - f(E) - float((dE.double() * step.double()).sum())) <= 800 * U * size


@gpu
def test_writing_in_place_is_seen_by_autograd():
    import torch
    from paper_2509_22418_b200 import ppu
    ids, it, dout, n = make(20, 16, 10)
    add = torch.randn(10, 16, device="cuda")
    before = add._version
    ppu.ppu_embed_bwd(it, dout, 10, add=add, in_place=True)
    assert add._version > before
    leaf = add.clone().requires_grad_()
    with pytest.raises(ppu.PpuError):
        ppu.ppu_embed_bwd(it, dout, 10, add=leaf, in_place=True)
    with torch.no_grad():
        ppu.ppu_embed_bwd(it, dout, 10, add=leaf, in_place=True)


# ---- refusals ----------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def ppu():
    from paper_2509_22418_b200 import build, ppu as mod
    build.build()
    return mod


F = ["ids", "E", "lde", "et", "scale", "out", "ldo", "ot", "T", "d", "V", "flags", "st"]
B = ["ids", "dout", "ldd", "dt", "scale", "add", "lda", "dE", "lde", "gt", "T", "d", "V", "ws", "nb", "flags", "st"]


def _call(fn, names, **change):
    buf = (C.c_uint8 * 65536)()
    base = (C.addressof(buf) + 255) & ~255
    a = {n: C.c_void_p(base) for n in names}
    a.update(scale=C.c_float(1.0), flags=None, st=None, T=4, d=64, V=10, nb=C.c_size_t(1 << 40), add=None)
    a.update({n: C.c_int64(64) for n in ("lde", "ldo", "ldd", "lda")}, et=0, ot=1, dt=1, gt=0)
    for n, x in change.items():
        a[n] = C.c_void_p(base + 4) if x == "odd" else C.c_void_p(base) if x == "there" else C.c_void_p(base + 1024) if x == "else" else x
    return fn(*[a[n] for n in names])


@pytest.mark.parametrize("change,code", [
    (dict(ids=None), -1), (dict(E=None), -1), (dict(out=None), -1), (dict(d=60), -2), (dict(d=16392), -2), (dict(d=0), -1), (dict(T=-1), -1), (dict(T=(1 << 20) + 1), -2),
    (dict(V=0), -1), (dict(V=(1 << 22) + 1), -2), (dict(lde=C.c_int64(56)), -1), (dict(ldo=C.c_int64(68)), -1), (dict(E="odd"), -1), (dict(out="odd"), -1), (dict(et=2), -1),
    (dict(ot=-1), -1),
])
def test_lookup_refuses(ppu, change, code):
    assert _call(ppu.lib().ppu_embed_fwd, F, **change) == code


@pytest.mark.parametrize("change,code", [
    (dict(ids=None), -1), (dict(dout=None), -1), (dict(dE=None), -1), (dict(ws=None), -1), (dict(nb=C.c_size_t(100)), -4), (dict(ws="odd"), -1), (dict(dout="odd"), -1),
    (dict(dE="odd"), -1), (dict(add="odd"), -1), (dict(d=20), -2), (dict(V=-3), -1), (dict(T=-1), -1), (dict(ldd=C.c_int64(60)), -1), (dict(lde=C.c_int64(32)), -1),
    (dict(add="else", lda=C.c_int64(63)), -1), (dict(add="there", lda=C.c_int64(128)), -1), (dict(dt=3), -1), (dict(gt=9), -1),
])
def test_gradient_refuses(ppu, change, code):
    assert _call(ppu.lib().ppu_embed_bwd, B, **change) == code


def test_workspace_sizes(ppu):
    assert ppu.ppu_embed_query_bytes(0, 64, 100) == 0
    for T, d, V in ((1, 8, 1), (8192, 2048, 32768), (1 << 20, 2048, 1 << 22)):
        assert 8 * T <= ppu.ppu_embed_query_bytes(T, d, V) <= 16 * T + 8 * d * 2112 + (4 << 20)
    for bad in ((-1, 8, 1), (1, 12, 1), (1, 8, 0), (1 << 31, 8, 1)):
        with pytest.raises(ppu.PpuError):
            ppu.ppu_embed_query_bytes(*bad)
    assert ppu.lib().ppu_embed_query_bytes(1, 8, 1, None) == -1


def test_words_and_tensors_are_checked(ppu):
    import torch
    ids, E = torch.zeros(4, dtype=torch.int32), torch.zeros(10, 64)
    for call in (lambda: ppu.ppu_embed_fwd(ids, E), lambda: ppu.ppu_embed_bwd(ids, E[:4], 10), lambda: ppu.ppu_embed_fwd(ids, E, dtype="fp16"),
                 lambda: ppu.ppu_embed_bwd(ids, E[:4], 10, dtype=torch.float32)):
        with pytest.raises(ppu.PpuError):
            call()


@gpu
def test_device_tensors_are_checked():
    import torch
    from paper_2509_22418_b200 import ppu
    c = dict(device="cuda")
    ids, E, g = torch.zeros(4, dtype=torch.int32, **c), torch.zeros(10, 64, **c), torch.zeros(4, 64, **c)
    for args in ((ids.long(), E), (ids.cpu(), E), (ids[None], E), (ids, E.half()), (ids, E[0]), (ids, E.t()), (ids, E[:, ::2]), (ids, torch.zeros(10, 60, **c))):
        with pytest.raises(ppu.PpuError):
            ppu.ppu_embed_fwd(*args)
    for args, kw in (((ids, g.half(), 10), {}), ((ids[:3], g, 10), {}), ((ids, g, 0), {}), ((ids, g, 10), dict(add=E[:9])), ((ids, g, 10), dict(add=E.half())),
                     ((ids, g, 10), dict(add=E, dtype="bf16")), ((ids, g, 10), dict(in_place=True)), ((ids, g, 10), dict(workspace=torch.zeros(64, dtype=torch.uint8, **c))),
                     ((ids, g, 1 << 40), {}), ((ids, g, 10), dict(flags=torch.zeros(7, dtype=torch.int32, **c)))):
        with pytest.raises(ppu.PpuError):
            ppu.ppu_embed_bwd(*args, **kw)
