"""8-bit products of few rows in every form that the rows' codes take (in memory, copied, quantised
by the kernel), very narrow ones, and both captured: bit for bit the oracle's."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _matrix(torch, rows, cols, seed):
    import paper_2202_06009_amd as zo
    g = torch.Generator().manual_seed(seed)
    q = zo.I8(rows, cols)
    codes = torch.zeros((rows, -(-cols // 128) * 128), dtype=torch.int8)
    codes[:, :cols] = torch.randint(-127, 128, (rows, cols), generator=g).to(torch.int8)
    q.codes.copy_(codes.view(-1))
    q.scales.copy_(torch.rand(rows, generator=g) * 2.0 ** -9)
    return q


def _codes(q):
    return q.codes.view(q.rows, -1)[:, :q.cols].double()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("m,n,k", [(32, 100, 6400), (20, 50, 8000), (29, 17, 131072), (16, 33, 7300),
                                   (32, 1, 1), (17, 515, 3584), (25, 2100, 4700)])
def test_few_rows(torch, m, n, k, dtype):
    import i8_ref as ref
    import paper_2202_06009_amd as zo
    a, b = _matrix(torch, m, k, 1), _matrix(torch, n, k, 2)
    out = torch.full((m, n + 3), 7.0, dtype=getattr(torch, dtype), device="cuda")
    zo.zo_i8_product(a, b, out[:, :n])
    assert torch.equal(out[:, :n], ref.product(_codes(a), a.scales, _codes(b), b.scales, out.dtype))
    assert bool((out[:, n:] == 7.0).all())


@pytest.mark.parametrize("m,n,k", [(33, 1, 1), (1000, 1, 129), (4097, 2, 640), (5000, 3, 200), (33, 5, 9000)])
def test_narrow(torch, m, n, k):
    import i8_ref as ref
    import paper_2202_06009_amd as zo
    a, b = _matrix(torch, m, k, 3), _matrix(torch, n, k, 4)
    out = torch.full((m, n + 1), 7.0, device="cuda")
    zo.zo_i8_product(a, b, out[:, :n])
    assert torch.equal(out[:, :n], ref.product(_codes(a), a.scales, _codes(b), b.scales, out.dtype))
    assert bool((out[:, n:] == 7.0).all())


@pytest.mark.parametrize("m,k", [(1, 1600), (4, 6400), (16, 4096), (30, 3712), (32, 6400)])
def test_captured(torch, m, k):
    """A decode step out of a graph, replayed with new activations between eager steps; two graphs
    with workspaces of their own in turn."""
    import paper_2202_06009_amd as zo
    n = 520
    w = _matrix(torch, n, k, 5)

    class Step:
        def __init__(self):
            self.x = torch.randn((m, k), device="cuda").bfloat16()
            self.xq, self.y = zo.I8(m, k), torch.empty((m, n), device="cuda")
            self.run()
            torch.cuda.synchronize()
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph):
                self.run()

        def run(self, y=None):
            zo.zo_i8_linear(self.x, w, self.y if y is None else y, self.xq)

    steps = [Step(), Step()]
    for i in range(4):
        for s in steps:
            s.x.copy_(torch.randn((m, k), device="cuda") * 2.0 ** i)
        for s in steps:
            s.graph.replay()
        torch.cuda.synchronize()
        for s in steps:
            want = torch.empty_like(s.y)
            s.run(want)
            assert torch.equal(s.y, want)
            s.y.fill_(7.0)
