"""The 8-bit, norm and log probability operators where offsets pass 32 bits and where the rows
take several launches: the same bits as on the rows by themselves."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    yield torch
    torch.cuda.empty_cache()


def _gen(torch):
    return torch.Generator(device="cuda").manual_seed(5)


def _apart(torch, rows, cols, ld, dtype, src=None):
    """[rows, cols] with row stride ld, in a buffer that ends with its last element."""
    t = torch.empty((rows - 1) * ld + cols, dtype=dtype, device="cuda").as_strided((rows, cols), (ld, 1))
    return t if src is None else t.copy_(src)


@pytest.mark.parametrize("ld", [2 ** 30, 2 ** 30 + 1])
def test_rows_far_apart(torch, ld):
    import paper_2202_06009_amd as zo
    rows, cols, bf16 = 5, 333, torch.bfloat16
    assert (rows - 1) * ld >= 2 ** 32
    x = torch.randn((rows, cols), device="cuda", generator=_gen(torch)).to(bf16)
    xf = _apart(torch, rows, cols, ld, bf16, x)
    yf = _apart(torch, rows, cols, ld, bf16)
    w = torch.randn(cols, device="cuda", generator=_gen(torch))
    work = torch.empty(1 << 16, device="cuda")

    def both(f):
        """f on the rows together and far apart, with buffers of their own for results."""
        near, far = f(x, torch.empty_like(x)), f(xf, yf)
        for a, b in zip(near, far):
            assert torch.equal(a, b)

    def quantised(x, y):
        q, qt = zo.I8(rows, cols), zo.I8(cols, rows)
        zo.zo_i8_quantize(x, q, qt, work)
        zo.zo_i8_dequantize(q, y)
        return q.codes, q.scales, qt.codes, qt.scales, y

    def multiplied(x, y):
        q, m, xq = zo.I8(rows, cols), zo.I8(cols, cols), zo.I8(rows, cols)
        zo.zo_i8_quantize(x.contiguous(), q)
        zo.zo_i8_quantize(torch.randn((cols, cols), device="cuda", generator=_gen(torch)), m)
        zo.zo_i8_product(q, m, y)
        first = y.clone()
        zo.zo_i8_linear(x, m, y, xq)
        return first, y

    def normed(x, y):
        rstd, dw, q = torch.empty(rows, device="cuda"), torch.empty_like(w), zo.I8(rows, cols)
        zo.zo_rms_norm(x, w, residual=x, out=y, q=q, rstd=rstd)
        first = y.clone()
        zo.zo_rms_norm_grad(x, x, w, rstd, y, dw, dh=x, work=work)
        second = y.clone()
        zo.zo_rms_norm_grad(x, x, w, rstd, y, dh=x)
        return first, q.codes, q.scales, rstd, second, dw, y

    def scored(x, y):
        tokens = torch.arange(rows, dtype=torch.int32, device="cuda")
        logp, stats = torch.empty(rows, device="cuda"), torch.empty((rows, 3), device="cuda")
        values = torch.empty((rows, 7), device="cuda")
        columns = torch.empty((rows, 7), dtype=torch.int32, device="cuda")
        zo.zo_token_logprobs(x, tokens, logp, stats, values, columns)
        zo.zo_token_logprobs_grad(x, stats, y, tokens=tokens, dlogp=logp, dentropy=logp)
        return logp, stats, values, columns, y

    for f in (quantised, multiplied, normed, scored):
        print(f.__name__, flush=True)
        both(f)


def test_product_rows_far_apart(torch):
    """Results of the tiled form, 40 rows 2^27 elements apart."""
    import paper_2202_06009_amd as zo
    rows, cols, ld = 40, 200, 2 ** 27
    x = torch.randn((rows, 333), device="cuda", generator=_gen(torch))
    m = torch.randn((cols, 333), device="cuda", generator=_gen(torch))
    q, mq = zo.I8(rows, 333), zo.I8(cols, 333)
    zo.zo_i8_quantize(x, q)
    zo.zo_i8_quantize(m, mq)
    near = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    far = _apart(torch, rows, cols, ld, torch.bfloat16)
    zo.zo_i8_product(q, mq, near)
    zo.zo_i8_product(q, mq, far)
    assert torch.equal(near, far)


@pytest.mark.parametrize("rows", [1, 40])
def test_codes_past_32_bits(torch, rows):
    """2^25 + 70 rows of 128 bytes, of which the last 70 are not zero."""
    import paper_2202_06009_amd as zo
    n, k, tail = 2 ** 25 + 70, 100, 70
    m = torch.zeros((n, k), dtype=torch.bfloat16, device="cuda")
    m[-tail:] = torch.randn((tail, k), device="cuda", generator=_gen(torch)).bfloat16()
    mq, some = zo.I8(n, k), zo.I8(tail, k)
    zo.zo_i8_quantize(m, mq)
    zo.zo_i8_quantize(m[-tail:], some)
    assert torch.equal(mq.codes[-tail * 128:], some.codes)
    assert torch.equal(mq.scales[-tail:], some.scales)
    x, q = torch.randn((rows, k), device="cuda", generator=_gen(torch)), zo.I8(rows, k)
    zo.zo_i8_quantize(x, q)
    out, want = torch.empty((rows, n), device="cuda"), torch.empty((rows, tail), device="cuda")
    zo.zo_i8_product(q, mq, out)
    zo.zo_i8_product(q, some, want)
    assert torch.equal(out[:, -tail:], want)
    assert not bool(out[:, :1000].any()) and not bool(out[:, -tail - 1000:-tail].any())
    zo.zo_i8_dequantize(mq, m)
    want = torch.empty((tail, k), dtype=m.dtype, device="cuda")
    zo.zo_i8_dequantize(some, want)
    assert torch.equal(m[-tail:], want)


def test_rows_of_several_launches(torch):
    import paper_2202_06009_amd as zo
    rows, cols, some = 2 ** 22 + 11, 24, 2 ** 21 - 5
    x = torch.randn((rows, cols), device="cuda", generator=_gen(torch))
    w = torch.randn(cols, device="cuda", generator=_gen(torch))

    def run(x):
        n = len(x)
        out, dx, dz, back = (torch.empty_like(x) for _ in range(4))
        q, codes = zo.I8(n, cols), zo.I8(n, cols)
        rstd, logp = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        stats, values = torch.empty((n, 3), device="cuda"), torch.empty((n, 3), device="cuda")
        columns = torch.empty((n, 3), dtype=torch.int32, device="cuda")
        tokens = (x[:, 0] * 100).int() % cols
        zo.zo_i8_quantize(x, codes)
        zo.zo_i8_dequantize(codes, back)
        zo.zo_rms_norm(x, w, residual=x, out=out, q=q, rstd=rstd)
        zo.zo_rms_norm_grad(out, x, w, rstd, dx, dh=x)
        zo.zo_token_logprobs(x, tokens, logp, stats, values, columns)
        zo.zo_token_logprobs_grad(x, stats, dz, tokens=tokens, dlogp=logp, dentropy=rstd)
        return (out, dx, dz, back, q.codes.view(n, 128), codes.codes.view(n, 128), q.scales,
                codes.scales, rstd, logp, stats, values, columns)

    whole = run(x)
    for at in (0, some, 2 * some):
        part = run(x[at:at + some])
        for a, b in zip(whole, part):
            assert torch.equal(a[at:at + some], b)
