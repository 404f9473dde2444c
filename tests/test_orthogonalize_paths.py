"""Further calls of the orthogonalised update (ppu_orthogonalize), by the way that their matrices take through the kernels: on chip (sides up to 128, a
cluster to a matrix), or step by step through memory on single SMs or SM pairs.  References and bounds are those of test_orthogonalize.py."""
import pytest

from test_orthogonalize import cuda, matrices, near

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
