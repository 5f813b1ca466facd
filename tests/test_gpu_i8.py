"""8-bit matrices on the GPU against the 64-bit oracle: codes, scales, values and
products bit for bit."""
import pytest

pytestmark = pytest.mark.gpu

DTYPES = ["float32", "float16", "bfloat16"]


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _input(torch, rows, cols, dtype, seed, pad=0):
    """Values of many magnitudes, whole rows of ties (multiples of half of the largest's
    127th part), zeros, inside a wider buffer whose other columns are NaN."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g)
    x = x * torch.exp2(torch.randint(-9, 9, (rows, 1), generator=g).float())
    ties = torch.randint(-254, 255, (rows, cols), generator=g).float() / 4
    ties[:, 0] = 63.5
    x = torch.where(torch.arange(rows)[:, None] % 3 == 1, ties, x)
    x = torch.where(torch.rand((rows, cols), generator=g) > 0.95, 0.0, x)
    full = torch.full((rows, cols + pad), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    full[:, :cols] = x.to(getattr(torch, dtype))
    return full[:, :cols]


def _quantized(torch, x, rows=True, cols=False):
    import paper_2202_06009_amd as zo
    r, c = x.shape
    out = []
    for want, (a, b) in ((rows, (r, c)), (cols, (c, r))):
        q = zo.I8(a, b) if want else None
        if q is not None:                       # whatever was there before must not matter
            q.codes.fill_(-1)
            q.scales.fill_(7.0)
        out.append(q)
    work = torch.empty(zo.zo_i8_work_bytes(r, c) // 4, device="cuda") if cols else None
    zo.zo_i8_quantize(x, *out, work)
    return out


def _check(torch, q, x):
    import i8_ref as ref
    codes, scales = ref.quantize(x.double())
    got = q.codes.view(q.rows, -1)
    assert torch.equal(got[:, :q.cols].double(), codes)
    assert not got[:, q.cols:].any()
    assert torch.equal(q.scales.isnan(), scales.isnan())
    assert torch.equal(q.scales.nan_to_num(0.0), scales.nan_to_num(0.0))


SHAPES = [(1, 1), (1, 31), (1, 127), (1, 128), (1, 129), (2, 255), (1, 1600), (3, 513), (15, 128),
          (17, 257), (64, 64), (65, 130), (127, 95), (129, 1601), (200, 40), (33, 2049),
          (513, 385), (5, 5000), (3, 20000), (700, 70)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_quantize(torch, shape, dtype):
    for pad, form in ((0, (True, True)), (1, (True, False)), (5, (False, True)), (8, (True, True))):
        x = _input(torch, *shape, dtype, seed=shape[0] * 31 + shape[1] + pad, pad=pad)
        q, qt = _quantized(torch, x, *form)
        if q is not None:
            _check(torch, q, x)
        if qt is not None:
            _check(torch, qt, x.t())


@pytest.mark.parametrize("shape,dtype", [((3, 40000), "float32"), ((2, 70001), "bfloat16"),
                                         ((20, 66000), "float16"), ((9000, 3), "bfloat16")])
def test_quantize_long(torch, shape, dtype):
    """Rows beyond a workgroup's registers; many short rows."""
    x = _input(torch, *shape, dtype, seed=9, pad=1)
    q, qt = _quantized(torch, x, True, True)
    _check(torch, q, x)
    _check(torch, qt, x.t())


@pytest.mark.parametrize("dtype", DTYPES)
def test_quantize_extremes(torch, dtype):
    """The type's largest and smallest values, steps below the normal numbers, NaN and
    infinities: rows and columns that they are not in do not notice."""
    dt = getattr(torch, dtype)
    info = torch.finfo(dt)
    x = torch.zeros((140, 300), dtype=dt, device="cuda")
    x[0, :3] = torch.tensor([info.max, info.min, info.max / 3])
    x[1, 5:9] = torch.tensor([info.tiny, info.tiny / 2, -info.tiny / 4, info.tiny / 128])
    x[2, 7] = info.smallest_normal * info.eps                # the smallest of all
    x[3, 11] = float("nan")
    x[4, 13] = float("inf")
    x[5, 17], x[5, 18] = -float("inf"), 1.0
    x[6, 20:] = -0.0
    x[7] = torch.arange(300, device="cuda").to(dt) / 7
    x[130] = x[7].flip(0)
    q, qt = _quantized(torch, x, True, True)
    _check(torch, q, x)
    _check(torch, qt, x.t())
    import paper_2202_06009_amd as zo
    out = torch.empty((140, 300), device="cuda")
    zo.zo_i8_dequantize(q, out)
    assert out[3:6].isnan().all() and int(out.isnan().any(1).sum()) == 3


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(1, 1), (3, 33), (5, 512), (66, 129), (130, 1601)])
def test_dequantize(torch, shape, dtype):
    import paper_2202_06009_amd as zo
    x = _input(torch, *shape, "float32", seed=5)
    q, _ = _quantized(torch, x)
    want = (q.codes.view(q.rows, -1)[:, :q.cols].float() * q.scales[:, None])
    for pad in (0, 3):
        full = torch.full((shape[0], shape[1] + pad), 7.0, dtype=getattr(torch, dtype),
                          device="cuda")
        zo.zo_i8_dequantize(q, full[:, :shape[1]])
        assert torch.equal(full[:, :shape[1]], want.to(full.dtype))
        assert (full[:, shape[1]:] == 7.0).all()


def _matrices(torch, m, n, k, seed):
    """Codes of the whole range, the largest ones throughout in some rows, and scales."""
    import paper_2202_06009_amd as zo
    g = torch.Generator().manual_seed(seed)
    got = []
    for rows in (m, n):
        q = zo.I8(rows, k)
        codes = torch.zeros((rows, -(-k // 128) * 128), dtype=torch.int8)
        codes[:, :k] = torch.randint(-127, 128, (rows, k), generator=g).to(torch.int8)
        codes[::3, :k] = 127
        codes[1::5, :k] = -127
        q.codes.copy_(codes.view(-1))
        q.scales.copy_(torch.rand(rows, generator=g) * 2.0 ** -9)
        got.append(q)
    return got


def _codes(q):
    return q.codes.view(q.rows, -1)[:, :q.cols].double()


PRODUCTS = [(1, 1, 1), (1, 16, 32), (2, 17, 31), (1, 100, 1600), (3, 65, 129), (8, 130, 127),
            (11, 515, 260), (16, 64, 128), (17, 64, 256), (31, 33, 640), (33, 31, 1153),
            (64, 64, 384), (65, 129, 500), (129, 70, 1000), (128, 256, 512), (256, 256, 1600),
            (257, 300, 999), (300, 520, 72), (511, 259, 4000), (640, 1000, 130), (1, 7, 131072),
            (70, 9, 131072), (1500, 2500, 300), (2047, 1024, 200)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("mnk", PRODUCTS)
def test_product(torch, mnk, dtype):
    import i8_ref as ref
    import paper_2202_06009_amd as zo
    m, n, k = mnk
    a, b = _matrices(torch, m, n, k, seed=m * 7 + n)
    want = ref.product(_codes(a), a.scales, _codes(b), b.scales, getattr(torch, dtype))
    for pad in (0, 1, 8):
        full = torch.full((m, n + pad), 7.0, dtype=getattr(torch, dtype), device="cuda")
        zo.zo_i8_product(a, b, full[:, :n])
        assert torch.equal(full[:, :n], want)
        assert (full[:, n:] == 7.0).all()


@pytest.mark.parametrize("m,n,k", [(2300, 7300, 200), (4090, 4100, 60), (2500, 7296, 1300),
                                   (3000, 6208, 2600), (300, 40000, 129)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_product_of_many_tiles(torch, m, n, k, dtype):
    import i8_ref as ref
    import paper_2202_06009_amd as zo
    a, b = _matrices(torch, m, n, k, seed=1)
    out = torch.full((m, n), 7.0, dtype=getattr(torch, dtype), device="cuda")
    zo.zo_i8_product(a, b, out)
    assert torch.equal(out, ref.product(_codes(a), a.scales, _codes(b), b.scales, out.dtype))


@pytest.mark.parametrize("m", [1, 2, 5, 8, 15, 16, 17, 33, 64, 65, 100])
@pytest.mark.parametrize("xdtype", DTYPES)
def test_linear(torch, m, xdtype):
    """Every count of rows around the forms for few, odd reduced lengths, strided
    activations; the rows' quantisation is that of zo_i8_quantize."""
    import i8_ref as ref
    import paper_2202_06009_amd as zo
    for n, k in ((48, 1601), (517, 64), (130, 6400), (1000, 31)):
        for out_dtype in (torch.float32, torch.bfloat16):
            x = _input(torch, m, k, xdtype, seed=m + n, pad=3)
            _, w = _matrices(torch, 1, n, k, seed=n)
            out = torch.full((m, n + 1), 7.0, dtype=out_dtype, device="cuda")
            zo.zo_i8_linear(x, w, out[:, :n], zo.I8(m, k))
            codes, scales = ref.quantize(x.double())
            assert torch.equal(out[:, :n], ref.product(codes, scales, _codes(w), w.scales, out_dtype))
            assert (out[:, n:] == 7.0).all()


def test_linear_nan_rows(torch):
    """A row with NaN or infinity gives a row of NaN, in the one-kernel form and the others,
    and leaves the other rows alone."""
    import paper_2202_06009_amd as zo
    _, w = _matrices(torch, 1, 40, 300, seed=3)
    for m in (4, 40, 100):
        x = torch.randn((m, 300), device="cuda")
        clean = torch.empty((m, 40), device="cuda")
        zo.zo_i8_linear(x, w, clean, zo.I8(m, 300))
        x[1, 299], x[3, 0] = float("nan"), float("-inf")
        out = torch.empty((m, 40), device="cuda")
        zo.zo_i8_linear(x, w, out, zo.I8(m, 300))
        bad = torch.zeros(m, dtype=torch.bool, device="cuda")
        bad[1] = bad[3] = True
        assert out[bad].isnan().all() and torch.equal(out[~bad], clean[~bad])


def test_empty(torch):
    import paper_2202_06009_amd as zo
    full = torch.full((4, 5), 7.0, device="cuda")
    zo.zo_i8_product(zo.I8(4, 0), zo.I8(5, 0), full)
    assert (full == 0).all()
    full = torch.full((100, 70), 7.0, device="cuda")
    nan = torch.full((100,), float("nan"), device="cuda")
    zo.zo_i8_product(zo.I8(100, 0, scales=nan), zo.I8(70, 0, scales=nan), full)
    assert (full == 0).all()
    zo.zo_i8_linear(torch.empty((4, 0), device="cuda"), zo.I8(70, 0), full[:4], zo.I8(4, 0))
    zo.zo_i8_product(zo.I8(0, 10), zo.I8(5, 10), torch.empty((0, 5), device="cuda"))
    zo.zo_i8_product(zo.I8(5, 10), zo.I8(0, 10), torch.empty((5, 0), device="cuda"))
    zo.zo_i8_quantize(torch.empty((0, 7), device="cuda"), zo.I8(0, 7), zo.I8(7, 0))
    zo.zo_i8_quantize(torch.empty((7, 0), device="cuda"), zo.I8(7, 0), zo.I8(0, 7))
    torch.cuda.synchronize()


def test_offsets_beyond_32_bits(torch):
    """Codes and results more than 2^32 bytes from their buffers' starts."""
    import i8_ref as ref
    import paper_2202_06009_amd as zo
    rows, cols = 70000, 65536
    codes = torch.zeros(rows * cols, dtype=torch.int8, device="cuda")
    scales = torch.ones(rows, device="cuda")
    x = torch.randn((3, cols), device="cuda").bfloat16()
    a = zo.I8(3, cols)
    zo.zo_i8_quantize(x, a)
    codes.view(rows, cols)[-3:] = a.codes.view(3, cols)
    w = zo.I8(rows, cols, codes, scales)
    out = torch.full((3, rows), 7.0, device="cuda")
    zo.zo_i8_product(a, w, out)
    assert (out[:, :-3] == 0).all()
    assert torch.equal(out[:, -3:], ref.product(_codes(a), a.scales, _codes(a),
                                                torch.ones(3, device="cuda"), out.dtype))
    many = zo.I8(100, cols)
    many.codes.copy_(codes[-100 * cols:])
    many.scales.fill_(0.5)
    out = torch.full((100, rows), 7.0, device="cuda")
    zo.zo_i8_product(many, w, out)
    assert (out[:, :-3] == 0).all()
    assert torch.equal(out[-3:, -3:], (_codes(a) @ _codes(a).t().contiguous()).float() * 0.5)
    tail = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    zo.zo_i8_dequantize(w, tail)
    assert torch.equal(tail[-3:].double(), _codes(a)) and not tail[:-3].any()


def test_streams_and_graph(torch):
    """A layer's training step on another stream and out of a graph, replayed with new inputs
    between eager work, equals the eager one bit for bit."""
    import paper_2202_06009_amd as zo
    t, n, k = 300, 520, 200
    x = torch.randn((t, k), device="cuda").bfloat16()
    w = torch.randn((n, k), device="cuda")
    dy = torch.randn((t, n), device="cuda").bfloat16()
    m = {name: zo.I8(*s) for name, s in dict(xq=(t, k), xt=(k, t), wq=(n, k), wt=(k, n), gq=(t, n),
                                             gt=(n, t)).items()}
    work = torch.empty(max(zo.zo_i8_work_bytes(*s) for s in ((t, k), (n, k), (t, n))) // 4,
                       device="cuda")

    def step(stream=None):
        y = torch.empty((t, n), dtype=torch.bfloat16, device="cuda")
        dx = torch.empty((t, k), device="cuda")
        dw = torch.empty((n, k), device="cuda")
        zo.zo_i8_quantize(x, m["xq"], m["xt"], work, stream=stream)
        zo.zo_i8_quantize(w, m["wq"], m["wt"], work, stream=stream)
        zo.zo_i8_product(m["xq"], m["wq"], y, stream=stream)
        zo.zo_i8_quantize(dy, m["gq"], m["gt"], work, stream=stream)
        zo.zo_i8_product(m["gq"], m["wt"], dx, stream=stream)
        zo.zo_i8_product(m["gt"], m["xt"], dw, stream=stream)
        return y, dx, dw

    eager = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = step(side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(eager, other):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        x.copy_(torch.randn((t, k), device="cuda"))
        dy.copy_(torch.randn((t, n), device="cuda") * 2.0 ** -i)
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in held]
        for a, b in zip(got, step()):
            assert torch.equal(a, b)
