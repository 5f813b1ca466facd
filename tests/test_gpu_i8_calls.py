"""What the Python binding of the 8-bit, norm and log probability operators refuses before
anything reaches the GPU; a matrix as both operands; rows behind a batch."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _raises(f, *args, **kw):
    with pytest.raises(ValueError):
        f(*args, **kw)


def test_i8_refusals(torch):
    import paper_2202_06009_amd as zo
    x = torch.randn((6, 300), device="cuda")
    q, qt, work = zo.I8(6, 300), zo.I8(300, 6), torch.empty(300, device="cuda")
    _raises(zo.zo_i8_quantize, x, q, qt)                               # no workspace
    _raises(zo.zo_i8_quantize, x, q, qt, work[:299])
    _raises(zo.zo_i8_quantize, x, q, qt, torch.empty(300))
    _raises(zo.zo_i8_quantize, x, work)
    _raises(zo.zo_i8_quantize, x.double(), q)
    _raises(zo.zo_i8_quantize, x.t(), qt)
    _raises(zo.zo_i8_quantize, x, zo.Mx4(6, 300))
    for bad in (zo.I8(6, 301), zo.I8(7, 300)):
        with pytest.raises(zo.ZoError):
            zo.zo_i8_quantize(x, bad)
    with pytest.raises(zo.ZoError):
        zo.zo_i8_quantize(x)
    with pytest.raises(zo.ZoError):                                    # codes off 16 bytes
        zo.zo_i8_quantize(x, zo.I8(6, 300, torch.empty(6 * 384 + 1, dtype=torch.int8,
                                                       device="cuda")[1:], torch.empty(6, device="cuda")))
    _raises(zo.I8, 6, 300, torch.empty(6 * 384 - 1, dtype=torch.int8, device="cuda"))
    _raises(zo.I8, 6, 300, None, torch.empty(5, device="cuda"))
    _raises(zo.I8, 6, 300, torch.empty(6 * 384, dtype=torch.uint8, device="cuda"))
    _raises(zo.zo_i8_product, q, q, torch.empty((6, 7), device="cuda"))
    with pytest.raises(zo.ZoError):
        zo.zo_i8_product(q, qt, torch.empty((6, 300), device="cuda"))
    _raises(zo.zo_i8_linear, x[:5], q, torch.empty((6, 6), device="cuda"), q)
    _raises(zo.zo_i8_dequantize, q, torch.empty((6, 299), device="cuda"))


def test_product_of_a_matrix_with_itself(torch):
    """The same bits as the plain form.  Not symmetric to the last bit: element (m, n) is
    RN(RN(S s(m)) s(n)) and (n, m) is RN(RN(S s(n)) s(m)), two roundings of half a step U each,
    so they differ by at most 4 U / (1 - 2 U), below 5 U, of the value."""
    import i8_ref as ref
    import paper_2202_06009_amd as zo
    x = torch.randn((6, 300), device="cuda")
    q = zo.I8(6, 300)
    zo.zo_i8_quantize(x, q)
    out = torch.empty((6, 6), device="cuda")
    zo.zo_i8_product(q, q, out)
    codes, scales = ref.quantize(x.double())
    assert torch.equal(out, ref.product(codes, scales, codes, scales, torch.float32))
    assert bool(((out - out.t()).double().abs() <= 5 * ref.U * out.double().abs()).all())


def test_norm_refusals(torch):
    import paper_2202_06009_amd as zo
    x, w = torch.randn((6, 40), device="cuda"), torch.ones(40, device="cuda")
    _raises(zo.zo_rms_norm, x, w[:39], out=x)
    _raises(zo.zo_rms_norm, x, w.bfloat16(), out=x)
    _raises(zo.zo_rms_norm, x, w, out=x.bfloat16())
    _raises(zo.zo_rms_norm, x, w, residual=x[:5], out=x)
    _raises(zo.zo_rms_norm, x, w, out=x, rstd=torch.empty(5, device="cuda"))
    _raises(zo.zo_rms_norm, x, w, q=zo.Mx4(6, 40))
    for kw in (dict(), dict(out=x, eps=0.0), dict(out=x, h=x), dict(q=zo.I8(6, 41))):
        with pytest.raises(zo.ZoError):
            zo.zo_rms_norm(x, w, **kw)
    r = torch.ones(6, device="cuda")
    _raises(zo.zo_rms_norm_grad, x, x, w, r, x, w.clone())             # no workspace
    _raises(zo.zo_rms_norm_grad, x, x, w, r, x, w.clone(), work=torch.empty(39, device="cuda"))
    _raises(zo.zo_rms_norm_grad, x, x.bfloat16(), w, r, x)
    _raises(zo.zo_rms_norm_grad, x, x, w, r[:5], x)
    with pytest.raises(zo.ZoError):
        zo.zo_rms_norm_grad(x, x, w, r)


def test_score_refusals(torch):
    import paper_2202_06009_amd as zo
    z = torch.randn((6, 40), device="cuda")
    tokens, logp = torch.zeros(6, dtype=torch.int32, device="cuda"), torch.empty(6, device="cuda")
    stats, values = torch.empty((6, 3), device="cuda"), torch.empty((6, 4), device="cuda")
    columns = torch.empty((6, 4), dtype=torch.int32, device="cuda")
    _raises(zo.zo_token_logprobs, z, tokens)
    _raises(zo.zo_token_logprobs, z, tokens.long(), logp)
    _raises(zo.zo_token_logprobs, z, tokens, logp[:5])
    _raises(zo.zo_token_logprobs, z, stats=stats[:, :2])
    _raises(zo.zo_token_logprobs, z, values=values)
    _raises(zo.zo_token_logprobs, z, columns=columns)
    _raises(zo.zo_token_logprobs, z, values=values, columns=columns.long())
    for kw in (dict(), dict(stats=stats, tau=0.0)):
        with pytest.raises(zo.ZoError):
            zo.zo_token_logprobs(z, **kw)
    wide = [torch.empty((6, 41), dtype=t, device="cuda") for t in (torch.float32, torch.int32)]
    with pytest.raises(zo.ZoError):
        zo.zo_token_logprobs(z, values=wide[0], columns=wide[1])
    _raises(zo.zo_token_logprobs_grad, z, stats, z.bfloat16(), dentropy=logp)
    _raises(zo.zo_token_logprobs_grad, z, stats, z[:, :39], dentropy=logp)
    for kw in (dict(), dict(dlogp=logp), dict(dentropy=logp, tau=float("nan"))):
        with pytest.raises(zo.ZoError):
            zo.zo_token_logprobs_grad(z, stats, z, **kw)


def test_padded_batch_leaves_what_is_behind_it(torch):
    """Rows behind the last sequence, in every buffer, stay as they were."""
    import paper_2202_06009_amd as zo
    x = torch.randn((9, 256), device="cuda").bfloat16()
    w = torch.ones(256, device="cuda")
    full = {n: torch.full((9, 256), 7.0, dtype=x.dtype, device="cuda") for n in ("h", "out", "dx")}
    rstd = torch.full((9,), 7.0, device="cuda")
    q = zo.I8(9, 256)
    q.codes.fill_(5)
    q.scales.fill_(7.0)
    part = zo.I8(6, 256, q.codes, q.scales)
    zo.zo_rms_norm(x[:6], w, residual=x[3:], h=full["h"][:6], out=full["out"][:6], q=part,
                   rstd=rstd[:6])
    zo.zo_rms_norm_grad(x[:6], full["h"][:6], w, rstd[:6], full["dx"][:6])
    assert all(bool((v[6:] == 7.0).all()) for v in full.values())
    assert bool((rstd[6:] == 7.0).all()) and bool((q.scales[6:] == 7.0).all())
    assert bool((q.codes[6 * 256:] == 5).all())
    stats, logp = torch.full((9, 3), 7.0, device="cuda"), torch.full((9,), 7.0, device="cuda")
    z = torch.randn((9, 256), device="cuda")
    zo.zo_token_logprobs(z[:6], torch.zeros(6, dtype=torch.int32, device="cuda"), logp[:6], stats[:6])
    assert bool((stats[6:] == 7.0).all()) and bool((logp[6:] == 7.0).all())
    before = z.clone()
    zo.zo_token_logprobs_grad(z[:6], stats[:6], z[:6], dentropy=logp[:6])
    assert torch.equal(z[6:], before[6:])
