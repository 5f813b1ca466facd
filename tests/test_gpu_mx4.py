"""4-bit matrices on the GPU against the 64-bit oracle: codes and scales bit for
bit in the stored layout, values exact, products within the bound that their
accumulation in binary32 and one rounding allow."""
import numpy as np
import pytest

import operators_ref as ref

pytestmark = pytest.mark.gpu

HALF_ULP = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _np(t):
    return t.double().cpu().numpy()


def _input(torch, rows, cols, dtype, seed, pad=0, special=True):
    """Values of all magnitudes of the type, with zero blocks, ties and signed
    zeros, inside a wider buffer whose other columns are NaN."""
    r = np.random.default_rng(seed)
    span = 100 if dtype != "float16" else 12
    x = r.normal(size=(rows, cols)) * np.exp2(r.integers(-span, span // 2, size=(rows, 1)))
    if special:
        pick = r.random(x.shape)
        scale = np.exp2(r.integers(-8, 3, size=(rows, cols)))
        x = np.where(pick < 0.3, r.integers(-32, 33, size=x.shape) / 4 * scale, x)
        x = np.where(pick > 0.95, 0.0, x)
        x = np.where(pick > 0.99, -0.0, x)
    full = torch.full((rows, cols + pad), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    full[:, :cols] = torch.from_numpy(x).to(getattr(torch, dtype))
    return full[:, :cols]


def _quantized(torch, x, rows=True, cols=True):
    import paper_2202_06009_amd as zo
    r, c = x.shape
    out = []
    for want, (a, b) in ((rows, (r, c)), (cols, (c, r))):
        q = zo.Mx4(a, b) if want else None
        if q is not None:                       # whatever was there before must not matter
            q.codes.fill_(0xFF)
            q.scales.fill_(0xFF)
        out.append(q)
    zo.zo_mx4_quantize(x, *out)
    return out


def _check_layout(q, x64):
    code, byte = ref.quantize(x64)
    codes, scales, dc, ds = ref.layout(code, byte, *x64.shape)
    gc, gs = q.codes.cpu().numpy(), q.scales.cpu().numpy()
    np.testing.assert_array_equal(gs[ds], scales[ds])
    np.testing.assert_array_equal(gc[dc], codes[dc])


SHAPES = [(1, 1), (1, 31), (1, 32), (1, 33), (2, 127), (1, 1600), (3, 129), (15, 128), (16, 256),
          (17, 257), (31, 7), (64, 64), (65, 130), (127, 95), (128, 128), (130, 1601), (200, 40),
          (300, 77), (513, 385)]


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_quantize_layout(torch, shape, dtype):
    for pad, form in ((0, (True, True)), (1, (True, False)), (5, (False, True)), (8, (True, True))):
        x = _input(torch, *shape, dtype, seed=shape[0] * 31 + shape[1] + pad, pad=pad)
        q, qt = _quantized(torch, x, *form)
        if q is not None:
            _check_layout(q, _np(x))
        if qt is not None:
            _check_layout(qt, _np(x).T)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_quantize_extremes(torch, dtype):
    """Largest and smallest values of the type, every midpoint, saturation, and
    blocks with NaN or infinities that leave their neighbours alone."""
    dt = getattr(torch, dtype)
    info = torch.finfo(dt)
    x = torch.zeros((4, 320), dtype=dt, device="cuda")
    x[0, 0], x[0, 32], x[0, 33] = info.max, info.tiny, info.smallest_normal
    x[0, 64] = info.smallest_normal * 2.0 ** -2            # below the normal numbers
    x[0, 96:104] = torch.tensor([.25, .75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.5])
    x[0, 128] = float("nan")
    x[0, 160] = float("inf")
    x[0, 193] = -float("inf")
    x[0, 224:256] = -0.0
    x[1] = -x[0]
    x[2] = info.min
    x[3, 300] = 1.0
    q, qt = _quantized(torch, x)
    _check_layout(q, _np(x))
    _check_layout(qt, _np(x).T)
    import paper_2202_06009_amd as zo
    out = torch.empty((4, 320), device="cuda")
    zo.zo_mx4_dequantize(q, out)
    np.testing.assert_array_equal(_np(out), ref.rounded(_np(x)))
    assert torch.isnan(out[0, 128:224]).all() and not torch.isnan(out[3]).any()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("shape", [(1, 1), (3, 33), (66, 129), (130, 1601)])
def test_dequantize(torch, shape, dtype):
    import paper_2202_06009_amd as zo
    x = _input(torch, *shape, "float16" if dtype == "float16" else "float32", seed=5)
    q, _ = _quantized(torch, x, cols=False)
    for pad in (0, 3):
        full = torch.full((shape[0], shape[1] + pad), 7.0, dtype=getattr(torch, dtype),
                          device="cuda")
        zo.zo_mx4_dequantize(q, full[:, :shape[1]])
        want = ref.rounded(_np(x))
        if dtype == "float16":
            want = want.astype(np.float16).astype(np.float64)
        np.testing.assert_array_equal(_np(full[:, :shape[1]]), want)
        assert (full[:, shape[1]:] == 7.0).all()


def _bound(a, b, dtype):
    """|error| of a b^T: K additions in binary32 (each at most 2^-23 of the sum of
    magnitudes, were they truncated) and the rounding of the result."""
    mag = np.abs(a) @ np.abs(b).T
    return (a.shape[1] + 8) * 2.0 ** -23 * mag, HALF_ULP[dtype]


def _check_product(out, a, b, dtype):
    want = a @ b.T
    acc, half = _bound(a, b, dtype)
    got = _np(out)
    tiny = 2.0 ** -25 if dtype == "float16" else 2.0 ** -134   # below the normal numbers
    assert (np.abs(got - want) <= acc + half * (np.abs(want) + acc) + tiny).all()


PRODUCTS = [(1, 1, 1), (1, 16, 32), (2, 17, 31), (1, 100, 1600), (3, 65, 129), (8, 130, 127),
            (11, 515, 260), (16, 64, 128), (17, 64, 256), (31, 33, 640), (33, 31, 1153),
            (64, 64, 384), (65, 129, 500), (129, 70, 1000), (128, 256, 512), (256, 256, 1600),
            (257, 300, 999), (300, 520, 72), (511, 259, 4000), (640, 1000, 130)]


@pytest.mark.parametrize("mnk", PRODUCTS)
def test_product_and_linear(torch, mnk):
    import paper_2202_06009_amd as zo
    m, n, k = mnk
    dtype = ["float32", "bfloat16", "float16"][sum(mnk) % 3]
    r = np.random.default_rng(m * 7 + n)
    # magnitudes that keep binary16 results finite
    xa = torch.from_numpy(r.normal(size=(m, k)) * np.exp2(r.integers(-6, 2, size=(m, 1))))
    xb = torch.from_numpy(r.normal(size=(n, k)) * np.exp2(r.integers(-6, 2, size=(n, 1))))
    xa, xb = xa.bfloat16().cuda(), xb.float().cuda()
    (a, _), (b, _) = _quantized(torch, xa, cols=False), _quantized(torch, xb, cols=False)
    va, vb = ref.rounded(_np(xa)), ref.rounded(_np(xb))
    for pad in (0, 1, 8):
        full = torch.full((m, n + pad), 7.0, dtype=getattr(torch, dtype), device="cuda")
        zo.zo_mx4_product(a, b, full[:, :n])
        _check_product(full[:, :n], va, vb, dtype)
        assert (full[:, n:] == 7.0).all()
        lin = torch.full((m, n + pad), 7.0, dtype=getattr(torch, dtype), device="cuda")
        zo.zo_mx4_linear(xa, b, lin[:, :n], zo.Mx4(m, k))
        _check_product(lin[:, :n], va, vb, dtype)
        assert (lin[:, n:] == 7.0).all()


@pytest.mark.parametrize("m,n,k", [(2300, 7300, 200), (4090, 4100, 60), (2050, 8200, 300),
                                   (2048, 17900, 60), (2000, 16300, 130), (6333, 1601, 1200),
                                   (2500, 7296, 1300), (4200, 4303, 1020),
                                   (3000, 6208, 2600)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_product_of_many_tiles(torch, m, n, k, dtype):
    """More tiles than the GPU has CUs, whole rounds of them and a rest; compared on
    the GPU in 64 bits."""
    import paper_2202_06009_amd as zo
    a = torch.randn((m, k), device="cuda")
    b = torch.randn((n, k), device="cuda")
    (aq, _), (bq, _) = _quantized(torch, a, cols=False), _quantized(torch, b, cols=False)
    va, vb = torch.empty_like(a), torch.empty_like(b)
    zo.zo_mx4_dequantize(aq, va)
    zo.zo_mx4_dequantize(bq, vb)
    out = torch.full((m, n), 7.0, dtype=getattr(torch, dtype), device="cuda")
    zo.zo_mx4_product(aq, bq, out)
    va, vb = va.double(), vb.double()
    want = va @ vb.t().contiguous()
    acc = (k + 8) * 2.0 ** -23 * (va.abs() @ vb.abs().t().contiguous())
    assert bool(((out.double() - want).abs()
                 <= acc + HALF_ULP[dtype] * (want.abs() + acc) + 2.0 ** -134).all())


@pytest.mark.parametrize("m", [1, 2, 5, 8, 15, 16, 17, 40, 64, 65, 100])
@pytest.mark.parametrize("xdtype", ["float32", "float16", "bfloat16"])
def test_linear_few_rows(torch, m, xdtype):
    """Every count of rows around the one-kernel form, over odd reduced lengths,
    strided activations and a long reduction."""
    import paper_2202_06009_amd as zo
    for n, k in ((48, 1601), (517, 64), (130, 6400), (1000, 31)):
        x = _input(torch, m, k, "float16", seed=m + k, pad=3).to(getattr(torch, xdtype))
        w = torch.from_numpy(np.random.default_rng(k).normal(size=(n, k))).float().cuda()
        wq, _ = _quantized(torch, w, cols=False)
        out = torch.full((m, n), 7.0, device="cuda")
        zo.zo_mx4_linear(x, wq, out, zo.Mx4(m, k))
        _check_product(out, ref.rounded(_np(x)), ref.rounded(_np(w)), "float32")


def test_empty_shapes(torch):
    import paper_2202_06009_amd as zo
    out = torch.full((3, 5), 7.0, device="cuda")
    zo.zo_mx4_product(zo.Mx4(3, 0), zo.Mx4(5, 0), out)      # a sum over nothing
    assert (out == 0).all()
    out.fill_(7.0)
    zo.zo_mx4_linear(torch.empty((3, 0), device="cuda"), zo.Mx4(5, 0), out, zo.Mx4(3, 0))
    assert (out == 0).all()
    zo.zo_mx4_product(zo.Mx4(0, 64), zo.Mx4(5, 64), torch.empty((0, 5), device="cuda"))
    zo.zo_mx4_quantize(torch.empty((0, 9), device="cuda"), zo.Mx4(0, 9), zo.Mx4(9, 0))
    zo.zo_mx4_dequantize(zo.Mx4(0, 9), torch.empty((0, 9), device="cuda"))


@pytest.mark.parametrize("m", [3, 40, 300])
def test_not_a_number_stays_in_its_row(torch, m):
    import paper_2202_06009_amd as zo
    x = torch.randn((m, 200), device="cuda")
    w = torch.randn((70, 200), device="cuda")
    x[1, 150], w[69, 0] = float("inf"), float("nan")
    (a, _), (b, _) = _quantized(torch, x, cols=False), _quantized(torch, w, cols=False)
    y, z = torch.empty((m, 70), device="cuda"), torch.empty((m, 70), device="cuda")
    zo.zo_mx4_product(a, b, y)
    zo.zo_mx4_linear(x, b, z, zo.Mx4(m, 200))
    want = torch.zeros((m, 70), dtype=torch.bool, device="cuda")
    want[1], want[:, 69] = True, True
    assert torch.equal(torch.isnan(y), want) and torch.equal(torch.isnan(z), want)


@pytest.mark.parametrize("t,n,k", [(1, 64, 96), (45, 70, 33), (130, 257, 160)])
def test_layer_backward(torch, t, n, k):
    """dx and dw against the formula, and against differences: the products are
    linear in the values their operands stand for, so a step along one of them
    changes sum(dy * y) by the gradient's sum exactly up to rounding."""
    import paper_2202_06009_amd as zo
    r = np.random.default_rng(t)
    x = torch.from_numpy(r.normal(size=(t, k))).bfloat16().cuda()
    w = torch.from_numpy(r.normal(size=(n, k)) * 0.05).float().cuda()
    dy = torch.from_numpy(r.normal(size=(t, n)) * 1e-3).bfloat16().cuda()
    (xq, xt), (wq, wt), (gq, gt) = (_quantized(torch, v) for v in (x, w, dy))
    dx, dw = torch.empty((t, k), device="cuda"), torch.empty((n, k), device="cuda")
    zo.zo_mx4_product(gq, wt, dx)
    zo.zo_mx4_product(gt, xt, dw)
    g, gT = ref.rounded(_np(dy)), ref.rounded(_np(dy).T)
    wT, xT = ref.rounded(_np(w).T), ref.rounded(_np(x).T)
    _check_product(dx, g, wT, "float32")
    _check_product(dw, gT, xT, "float32")
    # differences, with the weights of the transposed form: f(X) = sum(g * (X wT^T^T))
    def f(X):
        return float((g * (X @ wT)).sum())
    X, D = r.normal(size=(t, k)), r.normal(size=(t, k))
    slope = (f(X + 0.5 * D) - f(X - 0.5 * D))
    mag = (np.abs(g) @ np.abs(wT).T * np.abs(D)).sum()
    assert abs(float((_np(dx) * D).sum()) - slope) <= (n + 8) * 2.0 ** -23 * mag


def test_offsets_beyond_32_bits(torch):
    """More than 2^31 elements: the last rows land where the layout says."""
    import paper_2202_06009_amd as zo
    rows, cols = 66001, 33001
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    x[-70:] = torch.randn((70, cols), device="cuda").bfloat16()
    q = zo.Mx4(rows, cols)
    zo.zo_mx4_quantize(x, q)
    want = ref.rounded(_np(x[-70:]))
    out = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    zo.zo_mx4_dequantize(q, out)
    np.testing.assert_array_equal(_np(out[-70:]), want)
    assert not out[:1000].any()
    del out
    # the weights of a product: the last columns of its output, few rows and many
    for m in (2, 130):
        a = torch.randn((m, cols), device="cuda").bfloat16()
        aq, _ = _quantized(torch, a, cols=False)
        y = torch.empty((m, rows), device="cuda")
        zo.zo_mx4_product(aq, q, y)
        _check_product(y[:, -70:], ref.rounded(_np(a)), want, "float32")
        y.zero_()
        zo.zo_mx4_linear(a, q, y, zo.Mx4(m, cols))
        _check_product(y[:, -70:], ref.rounded(_np(a)), want, "float32")
    del q, y
    qt = zo.Mx4(cols, rows)
    zo.zo_mx4_quantize(x, None, qt)
    out = torch.empty((cols, rows), dtype=torch.bfloat16, device="cuda")
    zo.zo_mx4_dequantize(qt, out)
    lo = (rows - 70) // 32 * 32
    np.testing.assert_array_equal(_np(out[-9:, lo:]), ref.rounded(_np(x[lo:, -9:]).T))
    # output rows beyond 2^31 elements: long strides
    y = torch.empty((33000, 66000), device="cuda")[:, :200]
    a = torch.randn((33000, 64), device="cuda")
    b = torch.randn((200, 64), device="cuda")
    (aq, _), (bq, _) = _quantized(torch, a, cols=False), _quantized(torch, b, cols=False)
    zo.zo_mx4_product(aq, bq, y)
    _check_product(y[-40:], ref.rounded(_np(a[-40:])), ref.rounded(_np(b)), "float32")


@pytest.mark.parametrize("m", [2, 200])
def test_other_stream_and_graph(torch, m):
    """On a stream that is not the tensors' own, and recorded into a graph whose
    replays see new inputs."""
    import paper_2202_06009_amd as zo
    k, n = 300, 190
    x, w = torch.randn((m, k), device="cuda"), torch.randn((n, k), device="cuda")
    wq, xq = zo.Mx4(n, k), zo.Mx4(m, k)
    y = torch.empty((m, n), device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    zo.zo_mx4_quantize(w, wq, stream=s)
    zo.zo_mx4_linear(x, wq, y, xq, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    _check_product(y, ref.rounded(_np(x)), ref.rounded(_np(w)), "float32")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        zo.zo_mx4_quantize(w, wq)
        zo.zo_mx4_linear(x, wq, y, xq)
        zo.zo_mx4_quantize(x, xq)
        zo.zo_mx4_product(xq, wq, y)
    for i in range(4):
        x.normal_()
        w.mul_(1.7)
        y.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        _check_product(y, ref.rounded(_np(x)), ref.rounded(_np(w)), "float32")


def test_wrapper_refusals(torch):
    import paper_2202_06009_amd as zo
    x = torch.zeros((4, 40), device="cuda")
    q = zo.Mx4(4, 40)
    with pytest.raises(zo.ZoError) as e:
        zo.zo_mx4_quantize(x)
    assert e.value.status == zo.ZO_EINVAL
    with pytest.raises(zo.ZoError):
        zo.zo_mx4_quantize(x, zo.Mx4(4, 41))
    for bad in (x.double(), x.t(), x[0], x[0].expand(4, 40), x[:, ::2]):
        with pytest.raises(ValueError):
            zo.zo_mx4_quantize(bad, q)
    with pytest.raises(ValueError):
        zo.zo_mx4_product(q, q, torch.zeros((4, 5), device="cuda"))
    with pytest.raises(zo.ZoError):
        zo.zo_mx4_product(q, zo.Mx4(4, 39), torch.zeros((4, 4), device="cuda"))
    with pytest.raises(ValueError):
        zo.zo_mx4_linear(x[:3], q, torch.zeros((3, 4), device="cuda"), q)
    with pytest.raises(ValueError):
        zo.zo_mx4_product(q, "no matrix", x)
