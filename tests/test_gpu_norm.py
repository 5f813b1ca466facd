"""The root-mean-square norm and its gradients on the GPU against the 64-bit oracle: sums
and codes bit for bit, the rest within what its roundings allow (tests/i8_ref.py)."""
import pytest

pytestmark = pytest.mark.gpu

DTYPES = ["float32", "float16", "bfloat16"]
SHAPES = [(1, 1), (1, 2), (3, 7), (5, 128), (1, 1600), (9, 1601), (4, 511), (7, 513), (6, 1024),
          (3, 2047), (130, 260), (2, 4099), (3, 8192), (2, 16385), (1, 32768), (300, 100)]


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _buffer(torch, rows, cols, dtype, pad, fill=float("nan")):
    return torch.full((rows, cols + pad), fill, dtype=getattr(torch, dtype), device="cuda")


def _rows(torch, rows, cols, dtype, seed, pad=0, sigma=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g) * sigma
    x = torch.where(torch.rand((rows, cols), generator=g) < 0.02, 8 * x, x)
    full = _buffer(torch, rows, cols, dtype, pad)
    full[:, :cols] = x.to(full.dtype)
    return full[:, :cols]


def _weight(torch, cols, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (1 + 0.3 * torch.randn(cols, generator=g)).to(getattr(torch, dtype)).cuda()


def _within(torch, got, want, off, dtype):
    """|got - want| within off, the rounding to a type and what is below its normal numbers."""
    import i8_ref as ref
    half, tiny = ref.HALF[dtype], ref.TINY[dtype]
    err = (got.double() - want).abs()
    assert bool((err <= off + half * (want.abs() + off) + tiny).all()), float(
        (err - off - half * want.abs()).max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_norm(torch, shape, dtype):
    import i8_ref as ref
    import paper_2202_06009_amd as zo
    rows, cols = shape
    for i, (pad, res, wtype) in enumerate(((0, True, "float32"), (3, False, dtype),
                                           (8, True, dtype))):
        x = _rows(torch, rows, cols, dtype, seed=rows + cols + i, pad=pad)
        r = _rows(torch, rows, cols, dtype, seed=i, pad=pad + 1, sigma=3.0) if res else None
        w = _weight(torch, cols, wtype, seed=cols)
        h, out = (_buffer(torch, rows, cols, dtype, pad, 7.0) for _ in range(2))
        q, rstd = zo.I8(rows, cols), torch.empty(rows, device="cuda")
        q.codes.fill_(-1)
        zo.zo_rms_norm(x, w, residual=r, h=h[:, :cols], out=out[:, :cols], q=q, rstd=rstd, eps=1e-5)
        want_h = (x.float() + r.float()).to(x.dtype) if res else x
        assert torch.equal(h[:, :cols], want_h)
        assert (h[:, cols:] == 7.0).all() and (out[:, cols:] == 7.0).all()
        eps = float(torch.tensor(1e-5))
        want_rstd, want = ref.norm(want_h.double(), w.double(), eps)
        off = ref.rstd_off(cols)
        _within(torch, rstd, want_rstd, off * want_rstd, torch.float32)
        _within(torch, out[:, :cols], want, (off + 3 * ref.U) * want.abs(), x.dtype)
        codes, s = ref.quantize((want_h.float() * w.float()).double())
        got = q.codes.view(rows, -1)
        assert torch.equal(got[:, :cols].double(), codes) and not got[:, cols:].any()
        assert torch.equal(q.scales, s * rstd)
        # each output alone is the same
        for kw in (dict(out=torch.empty_like(out)[:, :cols]), dict(q=zo.I8(rows, cols)),
                   dict(h=torch.empty_like(h)[:, :cols]), dict(rstd=torch.empty_like(rstd))):
            zo.zo_rms_norm(x, w, residual=r, eps=1e-5, **kw)
            (name, v), = kw.items()
            if name == "q":
                assert torch.equal(v.codes, q.codes) and torch.equal(v.scales, q.scales)
            else:
                assert torch.equal(v, dict(out=out[:, :cols], h=h[:, :cols], rstd=rstd)[name])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols", [96, 1600, 5000])
def test_norm_extremes(torch, dtype, cols):
    """Rows of zeros, of the type's largest and of its smallest numbers (whose squares binary32
    does not hold), with NaN and infinities; their neighbours do not notice."""
    import i8_ref as ref
    import paper_2202_06009_amd as zo
    dt = getattr(torch, dtype)
    info = torch.finfo(dt)
    x = torch.randn((12, cols), device="cuda").to(dt)
    x[0] = 0.0
    x[1] = info.max
    x[1, ::2] = -info.max / 2
    x[2] = info.tiny
    x[2, 0] = -info.tiny * 64
    x[3, 5] = float("nan")
    x[4, 6] = float("inf")
    x[6] = x[6].float().mul(2.0 ** 70).to(dt)
    x[7] = x[7].float().mul(2.0 ** -100).to(dt)
    x[8] = 0.0
    x[8, cols - 1] = info.smallest_normal
    w = torch.ones(cols, device="cuda")
    w[::3] = 0.5
    fine = [i for i in range(12) if i not in (3, 4)]
    for eps in (2.0 ** -126, 2.0 ** -60, 1e-5, 1.0):
        out, rstd = torch.empty_like(x), torch.empty(12, device="cuda")
        q = zo.I8(12, cols)
        zo.zo_rms_norm(x, w, out=out, q=q, rstd=rstd, eps=eps)
        want_rstd, want = ref.norm(x.double(), w.double(), float(torch.tensor(eps)))
        off = ref.rstd_off(cols) + 4 * ref.U
        _within(torch, rstd[fine], want_rstd[fine], off * want_rstd[fine], torch.float32)
        _within(torch, out[fine], want[fine], (off + 4 * ref.U) * want[fine].abs(), dt)
        codes, s = ref.quantize((x.float() * w).double())
        got = q.codes.view(12, -1)[:, :cols].double()
        assert torch.equal(got, codes)
        assert torch.equal(q.scales[fine], (s * rstd)[fine])
        assert rstd[3].isnan() and rstd[4] == 0 and q.scales[3:5].isnan().all()
        assert out[3].isnan().all() and out[4, 6].isnan() and not out[4, :6].any()
        assert not out[0].any() and q.scales[0] == 0


def test_norm_in_place(torch):
    """h in the place of x or of the residual, out in the other's."""
    import paper_2202_06009_amd as zo
    for cols in (1600, 4100):
        x, r = (_rows(torch, 37, cols, "bfloat16", seed=s, pad=5) for s in (1, 2))
        w = _weight(torch, cols, "float32", seed=3)
        h, out = (torch.empty((37, cols), dtype=x.dtype, device="cuda") for _ in range(2))
        zo.zo_rms_norm(x, w, residual=r, h=h, out=out)
        for swap in (False, True):
            a, b = (v.clone(memory_format=torch.preserve_format) for v in (x, r))
            zo.zo_rms_norm(a, w, residual=b, h=b if swap else a, out=a if swap else b)
            got_h, got = (b, a) if swap else (a, b)
            assert torch.equal(got_h, h) and torch.equal(got, out)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES + [(1000, 70), (2100, 33), (257, 1600), (40, 9000)])
def test_norm_grad(torch, shape, dtype):
    import i8_ref as ref
    import paper_2202_06009_amd as zo
    rows, cols = shape
    for i, (pad, with_dh, wtype) in enumerate(((0, True, "float32"), (3, False, dtype))):
        h = _rows(torch, rows, cols, dtype, seed=rows + i, pad=pad, sigma=2.0)
        dy = _rows(torch, rows, cols, dtype, seed=cols + i, pad=pad + 2, sigma=2.0 ** -6)
        dh = _rows(torch, rows, cols, dtype, seed=i, pad=1, sigma=2.0 ** -5) if with_dh else None
        w = _weight(torch, cols, wtype, seed=cols)
        rstd = ref.norm(h.double(), w.double(), 1e-5)[0].float()
        dx, dw = _buffer(torch, rows, cols, dtype, pad, 7.0), torch.full((cols,), 7.0, device="cuda")
        work = torch.full((zo.zo_rms_norm_work_bytes(rows, cols) // 4,), float("nan"), device="cuda")
        zo.zo_rms_norm_grad(dy, h, w, rstd, dx[:, :cols], dw, dh=dh, work=work)
        want, want_dw, off, off_dw = ref.norm_grad(dy.double(), h.double(), w.double(),
                                                   rstd.double(), None if dh is None else dh.double())
        _within(torch, dx[:, :cols], want, off, h.dtype)
        _within(torch, dw, want_dw, off_dw, torch.float32)
        assert (dx[:, cols:] == 7.0).all()
        # either alone, and dx in the place of an input, is the same
        alone = torch.empty_like(dw)
        zo.zo_rms_norm_grad(dy, h, w, rstd, None, alone, dh=dh, work=work)
        assert torch.equal(alone, dw)
        for name in ("dy", "h", "dh"):
            args = dict(dy=dy, h=h, dh=dh)
            if args[name] is not None:
                args[name] = args[name].clone(memory_format=torch.preserve_format)
                zo.zo_rms_norm_grad(args["dy"], args["h"], w, rstd, args[name], dh=args["dh"])
                assert torch.equal(args[name], dx[:, :cols])


def test_norm_grad_by_differences(torch):
    """The gradients of a smooth function of out against differences of the norm itself, in
    binary32: a central difference over 2^-7 of the inputs' size has a relative error of
    about 2^-14 from the third derivative and 2^-16 from the roundings."""
    import paper_2202_06009_amd as zo
    rows, cols, eps = 5, 33, 1e-3
    x, r = torch.randn((rows, cols), device="cuda"), torch.randn((rows, cols), device="cuda")
    w, mix = torch.rand(cols, device="cuda") + 0.5, torch.randn((rows, cols), device="cuda")

    def value(x, r, w):
        out, h = torch.empty_like(x), torch.empty_like(x)
        zo.zo_rms_norm(x, w, residual=r, h=h, out=out, eps=eps)
        return float((out.double() * mix.double()).sum() + (h.double() * 0.25).sum())

    h, rstd = torch.empty_like(x), torch.empty(rows, device="cuda")
    zo.zo_rms_norm(x, w, residual=r, h=h, rstd=rstd, eps=eps)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    work = torch.empty(zo.zo_rms_norm_work_bytes(rows, cols) // 4, device="cuda")
    zo.zo_rms_norm_grad(mix, h, w, rstd, dx, dw, dh=torch.full_like(x, 0.25), work=work)
    for which, grad in ((0, dx), (1, dx), (2, dw)):
        along = torch.randn_like(grad)
        ends = []
        for sign in (1, -1):
            args = [x, r, w]
            args[which] = args[which] + sign * 2.0 ** -7 * along
            ends.append(value(*args))
        got = (ends[0] - ends[1]) * 2.0 ** 6
        want = float((grad.double() * along.double()).sum())
        size = float((grad.double() * along.double()).abs().sum())
        assert abs(got - want) <= 2.0 ** -10 * size


def test_norm_empty_and_large(torch):
    import paper_2202_06009_amd as zo
    w, dw = torch.ones(40, device="cuda"), torch.full((40,), 7.0, device="cuda")
    none = torch.empty((0, 40), device="cuda")
    zo.zo_rms_norm(none, w, out=none.clone(), q=zo.I8(0, 40))
    zo.zo_rms_norm(none, w, out=none.clone())
    zo.zo_rms_norm_grad(none, none, w, torch.empty(0, device="cuda"), none.clone())
    zo.zo_rms_norm_grad(none, none, w, torch.empty(0, device="cuda"), none.clone(), dw)
    assert (dw == 0).all()
    # offsets beyond 2^32 bytes
    x = torch.zeros((1 << 19, 4352), dtype=torch.bfloat16, device="cuda")
    x[-2:] = torch.randn((2, 4352), device="cuda")
    w = torch.rand(4352, device="cuda")
    out = torch.empty_like(x)
    zo.zo_rms_norm(x, w, out=out)
    small = torch.empty_like(out[-2:])
    zo.zo_rms_norm(x[-2:].clone(), w, out=small)
    assert torch.equal(out[-2:], small) and not out[:-2].any()


def test_norm_stream_and_graph(torch):
    import paper_2202_06009_amd as zo
    rows, cols = 200, 1600
    x, r = (torch.randn((rows, cols), device="cuda").bfloat16() for _ in range(2))
    w, q = torch.rand(cols, device="cuda"), zo.I8(rows, cols)
    work = torch.empty(zo.zo_rms_norm_work_bytes(rows, cols) // 4, device="cuda")

    def step(stream=None):
        h, out, dx = (torch.empty_like(x) for _ in range(3))
        rstd, dw = torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda")
        zo.zo_rms_norm(x, w, residual=r, h=h, out=out, q=q, rstd=rstd, stream=stream)
        zo.zo_rms_norm_grad(out, h, w, rstd, dx, dw, dh=h, work=work, stream=stream)
        return h, out, rstd, dx, dw

    eager = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        x.copy_(torch.randn((rows, cols), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in held] + [q.codes.clone()]
        assert all(torch.equal(a, b) for a, b in zip(got, list(step()) + [q.codes]))
