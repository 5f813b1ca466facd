"""Refusals and sizes of the 8-bit, norm and log probability operators: no kernel is
launched."""
import ctypes

import pytest

import paper_2202_06009_amd as zo

P = 1 << 20        # stands for a device pointer in calls that are refused
NAN, INF = float("nan"), float("inf")


def _i8(rows, cols, codes=P, scales=P):
    return zo._I8(codes, scales, rows, cols)


def _ref(x):
    return None if x is None else ctypes.byref(x)


def test_sizes():
    assert zo.zo_i8_code_bytes(0, 5) == 0 and zo.zo_i8_code_bytes(5, 0) == 0
    assert zo.zo_i8_code_bytes(3, 1) == 384 and zo.zo_i8_code_bytes(7, 1600) == 7 * 1664
    assert zo.zo_i8_code_bytes(1 << 20, 1 << 16) == 1 << 36           # past 32 bits
    assert zo.zo_i8_work_bytes(0, 9) == 0 and zo.zo_i8_work_bytes(1, 9) == 36
    for rows in (1, 15, 16, 17, 1000, 8192, 100000, 1 << 30):
        blocks = zo.zo_i8_work_bytes(rows, 1) // 4
        assert 1 <= blocks <= min(512, (rows + 15) // 16)
    for rows in (1, 64, 1000, 8192, 100000):
        blocks = zo.zo_rms_norm_work_bytes(rows, 1) // 4
        assert 1 <= blocks <= min(512, rows, 64 + rows // 16)
    assert zo.zo_rms_norm_work_bytes(0, 5) == 0
    for f, bad in ((zo.zo_i8_code_bytes, (-1, 1)), (zo.zo_i8_code_bytes, (1, (1 << 30) + 1)),
                   (zo.zo_i8_work_bytes, (1, -1)), (zo.zo_rms_norm_work_bytes, (-1, 1)),
                   (zo.zo_rms_norm_work_bytes, (1, 0)), (zo.zo_rms_norm_work_bytes, (1, 32769))):
        with pytest.raises(zo.ZoError) as e:
            f(*bad)
        assert e.value.status == zo.ZO_EINVAL


@pytest.mark.parametrize("over,code", [
    (dict(dtype=3), zo.ZO_EINVAL), (dict(dtype=-1), zo.ZO_EINVAL),
    (dict(x=None), zo.ZO_EINVAL), (dict(rows=-1), zo.ZO_EINVAL), (dict(ld=9), zo.ZO_EINVAL),
    (dict(x=P + 2), zo.ZO_EALIGN), (dict(dtype=1, x=P + 1), zo.ZO_EALIGN),
    (dict(q=None), zo.ZO_EINVAL), (dict(q=_i8(4, 11)), zo.ZO_EINVAL),
    (dict(qt=_i8(4, 10)), zo.ZO_EINVAL), (dict(q=_i8(4, 10, codes=None)), zo.ZO_EINVAL),
    (dict(q=_i8(4, 10, scales=None)), zo.ZO_EINVAL),
    (dict(q=_i8(4, 10, codes=P + 8)), zo.ZO_EALIGN),
    (dict(q=_i8(4, 10, scales=P + 2)), zo.ZO_EALIGN),
    (dict(qt=_i8(10, 4), work=None), zo.ZO_EINVAL),
    (dict(qt=_i8(10, 4), work=P + 1), zo.ZO_EALIGN),
    (dict(rows=0, q=_i8(0, 10), x=None), zo.ZO_OK),
    (dict(cols=0, ld=0, q=_i8(4, 0, None, None), qt=_i8(0, 4), x=None, work=None), zo.ZO_OK),
])
def test_quantize_refusals(over, code):
    a = dict(x=P, dtype=0, rows=4, cols=10, ld=10, q=_i8(4, 10), qt=None, work=P)
    a.update(over)
    assert zo.lib().zo_i8_quantize(a["x"], a["dtype"], a["rows"], a["cols"], a["ld"], _ref(a["q"]),
                                   _ref(a["qt"]), a["work"], None) == code


@pytest.mark.parametrize("a,b,out,dtype,ld,code", [
    (_i8(4, 10), _i8(5, 11), P, 0, 5, zo.ZO_EINVAL),       # reduced axes differ
    (_i8(4, 131073), _i8(5, 131073), P, 0, 5, zo.ZO_EINVAL),   # sums beyond 32 bits
    (_i8(4, 10), _i8(5, 10), None, 0, 5, zo.ZO_EINVAL),
    (_i8(4, 10), _i8(5, 10), P, 7, 5, zo.ZO_EINVAL),
    (_i8(4, 10), _i8(5, 10), P, 0, 4, zo.ZO_EINVAL),
    (_i8(4, 10), _i8(5, 10), P + 1, 2, 5, zo.ZO_EALIGN),
    (_i8(4, 10, codes=None), _i8(5, 10), P, 0, 5, zo.ZO_EINVAL),
    (_i8(4, 10), _i8(5, 10, codes=P + 4), P, 0, 5, zo.ZO_EALIGN),
    (None, _i8(5, 10), P, 0, 5, zo.ZO_EINVAL), (_i8(4, 10), None, P, 0, 5, zo.ZO_EINVAL),
    (_i8(0, 10), _i8(5, 10), None, 0, 5, zo.ZO_OK),
])
def test_product_refusals(a, b, out, dtype, ld, code):
    L = zo.lib()
    assert L.zo_i8_product(_ref(a), _ref(b), out, dtype, ld, None) == code
    if a is not None:
        assert L.zo_i8_linear(P, 0, max(1, a.cols), _ref(b), _ref(a), out, dtype, ld,
                              None) == code
    if code == zo.ZO_EINVAL and a is not None and b is not None and a.cols == b.cols <= 131072:
        assert L.zo_i8_linear(None, 0, a.cols, _ref(b), _ref(a), P, 0, 5, None) == zo.ZO_EINVAL


def test_dequantize_refusals():
    L = zo.lib()
    assert L.zo_i8_dequantize(None, P, 0, 10, None) == zo.ZO_EINVAL
    assert L.zo_i8_dequantize(_ref(_i8(4, 10)), None, 0, 10, None) == zo.ZO_EINVAL
    assert L.zo_i8_dequantize(_ref(_i8(4, 10)), P, 0, 9, None) == zo.ZO_EINVAL
    assert L.zo_i8_dequantize(_ref(_i8(4, 10)), P, 5, 10, None) == zo.ZO_EINVAL
    assert L.zo_i8_dequantize(_ref(_i8(4, 10)), P + 2, 0, 10, None) == zo.ZO_EALIGN
    assert L.zo_i8_dequantize(_ref(_i8(0, 10)), None, 0, 10, None) == zo.ZO_OK


def test_matrices_beyond_a_launch_are_refused():
    L, most = zo.lib(), 1 << 30
    assert L.zo_i8_quantize(P, 2, most, 129, 129, None, _ref(_i8(129, most)), P, None) == zo.ZO_EINVAL
    assert L.zo_i8_product(_ref(_i8(1, 10)), _ref(_i8(most, 10)), P, 2, most, None) == zo.ZO_EINVAL
    assert L.zo_i8_product(_ref(_i8(most, 10)), _ref(_i8(most, 10)), P, 2, most,
                           None) == zo.ZO_EINVAL


NORM = dict(x=P, dtype=2, rows=4, cols=10, ldx=10, residual=P, ldr=10, weight=P, weight_dtype=0,
            eps=1e-5, h=2 * P, ldh=10, out=3 * P, ldo=10, q=None, rstd=P)


@pytest.mark.parametrize("over,code", [
    (dict(dtype=3), zo.ZO_EINVAL), (dict(weight_dtype=1), zo.ZO_EINVAL),
    (dict(weight_dtype=-1), zo.ZO_EINVAL), (dict(dtype=0, weight_dtype=2), zo.ZO_EINVAL),
    (dict(rows=-1), zo.ZO_EINVAL), (dict(rows=1 << 31), zo.ZO_EINVAL), (dict(cols=0), zo.ZO_EINVAL),
    (dict(cols=32769, ldx=40000, ldr=40000, ldh=40000, ldo=40000), zo.ZO_EINVAL),
    (dict(eps=0.0), zo.ZO_EINVAL), (dict(eps=-1.0), zo.ZO_EINVAL), (dict(eps=NAN), zo.ZO_EINVAL),
    (dict(eps=INF), zo.ZO_EINVAL), (dict(eps=2.0 ** -127), zo.ZO_EINVAL),
    (dict(x=None), zo.ZO_EINVAL), (dict(weight=None), zo.ZO_EINVAL), (dict(ldx=9), zo.ZO_EINVAL),
    (dict(ldr=9), zo.ZO_EINVAL), (dict(ldh=9), zo.ZO_EINVAL), (dict(ldo=9), zo.ZO_EINVAL),
    (dict(h=None, out=None, rstd=None), zo.ZO_EINVAL), (dict(h=3 * P), zo.ZO_EINVAL),
    (dict(x=P, h=P, ldh=11), zo.ZO_EINVAL), (dict(residual=5 * P, out=5 * P, ldo=12), zo.ZO_EINVAL),
    (dict(q=_i8(4, 11)), zo.ZO_EINVAL), (dict(q=_i8(4, 10, codes=None)), zo.ZO_EINVAL),
    (dict(q=_i8(4, 10, codes=P + 8)), zo.ZO_EALIGN), (dict(x=P + 1), zo.ZO_EALIGN),
    (dict(weight=P + 2), zo.ZO_EALIGN), (dict(rstd=P + 2), zo.ZO_EALIGN),
    (dict(out=P + 1), zo.ZO_EALIGN), (dict(rows=0, x=None, weight=None), zo.ZO_OK),
])
def test_norm_refusals(over, code):
    a = {**NORM, **over}
    if a["q"] is not None:
        a["q"] = ctypes.addressof(a["q"])
    assert zo.lib().zo_rms_norm(ctypes.byref(zo._Norm(**a)), None) == code


BACK = dict(dy=P, dtype=2, rows=4, cols=10, lddy=10, h=2 * P, ldh=10, weight=P, weight_dtype=0,
            rstd=P, dh=3 * P, lddh=10, dx=4 * P, lddx=10, dw=P, work=P)


@pytest.mark.parametrize("over,code", [
    (dict(dtype=3), zo.ZO_EINVAL), (dict(weight_dtype=1), zo.ZO_EINVAL),
    (dict(rows=-1), zo.ZO_EINVAL), (dict(cols=0), zo.ZO_EINVAL), (dict(dx=None, dw=None), zo.ZO_EINVAL),
    (dict(dy=None), zo.ZO_EINVAL), (dict(h=None), zo.ZO_EINVAL), (dict(weight=None), zo.ZO_EINVAL),
    (dict(rstd=None), zo.ZO_EINVAL), (dict(work=None), zo.ZO_EINVAL), (dict(lddy=9), zo.ZO_EINVAL),
    (dict(ldh=9), zo.ZO_EINVAL), (dict(lddh=9), zo.ZO_EINVAL), (dict(lddx=9), zo.ZO_EINVAL),
    (dict(dx=P, lddx=11), zo.ZO_EINVAL), (dict(dx=2 * P, lddx=11), zo.ZO_EINVAL),
    (dict(dx=3 * P, lddx=11), zo.ZO_EINVAL), (dict(dy=P + 1), zo.ZO_EALIGN),
    (dict(dw=P + 2), zo.ZO_EALIGN), (dict(work=P + 2), zo.ZO_EALIGN),
    (dict(rstd=P + 2), zo.ZO_EALIGN), (dict(weight=P + 2), zo.ZO_EALIGN),
    (dict(rows=0, dw=None, dy=None), zo.ZO_OK),
])
def test_norm_grad_refusals(over, code):
    assert zo.lib().zo_rms_norm_grad(ctypes.byref(zo._NormBack(**{**BACK, **over})), None) == code


SCORE = dict(z=P, dtype=2, rows=4, vocab=10, ldz=10, tokens=P, tau=1.0, logp=P, stats=P, top=2,
             values=P, columns=P)


@pytest.mark.parametrize("over,code", [
    (dict(dtype=3), zo.ZO_EINVAL), (dict(rows=-1), zo.ZO_EINVAL), (dict(vocab=0), zo.ZO_EINVAL),
    (dict(vocab=1 << 31, ldz=1 << 31), zo.ZO_EINVAL), (dict(ldz=9), zo.ZO_EINVAL),
    (dict(z=None), zo.ZO_EINVAL), (dict(top=-1), zo.ZO_EINVAL), (dict(top=11), zo.ZO_EINVAL),
    (dict(top=1025, vocab=5000, ldz=5000), zo.ZO_EINVAL), (dict(logp=None), zo.ZO_EINVAL),
    (dict(values=None), zo.ZO_EINVAL), (dict(columns=None), zo.ZO_EINVAL),
    (dict(tokens=None, stats=None, top=0), zo.ZO_EINVAL), (dict(tau=0.0), zo.ZO_EINVAL),
    (dict(tau=-1.0), zo.ZO_EINVAL), (dict(tau=NAN), zo.ZO_EINVAL), (dict(tau=INF), zo.ZO_EINVAL),
    (dict(tau=2.0 ** -127), zo.ZO_EINVAL), (dict(z=P + 1), zo.ZO_EALIGN),
    (dict(tokens=P + 2), zo.ZO_EALIGN), (dict(logp=P + 2), zo.ZO_EALIGN),
    (dict(stats=P + 2), zo.ZO_EALIGN), (dict(values=P + 2), zo.ZO_EALIGN),
    (dict(columns=P + 2), zo.ZO_EALIGN), (dict(rows=0, z=None), zo.ZO_OK),
])
def test_score_refusals(over, code):
    assert zo.lib().zo_token_logprobs(ctypes.byref(zo._Score(**{**SCORE, **over})), None) == code


SCORE_BACK = dict(z=P, dtype=2, rows=4, vocab=10, ldz=10, tokens=P, stats=P, tau=1.0, dlogp=P,
                  dentropy=P, dz=2 * P, lddz=10)


@pytest.mark.parametrize("over,code", [
    (dict(dtype=3), zo.ZO_EINVAL), (dict(rows=-1), zo.ZO_EINVAL), (dict(vocab=0), zo.ZO_EINVAL),
    (dict(ldz=9), zo.ZO_EINVAL), (dict(lddz=9), zo.ZO_EINVAL), (dict(z=None), zo.ZO_EINVAL),
    (dict(dz=None), zo.ZO_EINVAL), (dict(stats=None), zo.ZO_EINVAL),
    (dict(dlogp=None, dentropy=None), zo.ZO_EINVAL), (dict(tokens=None), zo.ZO_EINVAL),
    (dict(dz=P, lddz=11), zo.ZO_EINVAL), (dict(tau=0.0), zo.ZO_EINVAL), (dict(tau=NAN), zo.ZO_EINVAL),
    (dict(z=P + 1), zo.ZO_EALIGN), (dict(dz=P + 1), zo.ZO_EALIGN), (dict(stats=P + 2), zo.ZO_EALIGN),
    (dict(tokens=P + 2), zo.ZO_EALIGN), (dict(dlogp=P + 2), zo.ZO_EALIGN),
    (dict(dentropy=P + 2), zo.ZO_EALIGN), (dict(rows=0, z=None, dz=None), zo.ZO_OK),
])
def test_score_grad_refusals(over, code):
    assert zo.lib().zo_token_logprobs_grad(ctypes.byref(zo._ScoreBack(**{**SCORE_BACK, **over})),
                                           None) == code


def test_null_arguments():
    L = zo.lib()
    for f in (L.zo_rms_norm, L.zo_rms_norm_grad, L.zo_token_logprobs, L.zo_token_logprobs_grad):
        assert f(None, None) == zo.ZO_EINVAL


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros((2, 4))
    with pytest.raises(ValueError):
        zo.zo_rms_norm(x, torch.ones(4), out=x.clone())
    with pytest.raises(ValueError):
        zo.zo_rms_norm_grad(x, x, torch.ones(4), torch.ones(2), x.clone())
    with pytest.raises(ValueError):
        zo.zo_token_logprobs(x, stats=torch.zeros((2, 3)))
    with pytest.raises(ValueError):
        zo.zo_token_logprobs_grad(x, torch.zeros((2, 3)), x.clone(), dentropy=torch.zeros(2))
    with pytest.raises(ValueError):
        zo.zo_i8_quantize(x)
    with pytest.raises(ValueError):
        zo.I8(2, 4, device="cpu")
    with pytest.raises(ValueError):
        zo.I8(2, 4, torch.zeros(256), torch.zeros(2))


def test_oracle_by_hand():
    """The oracle on numbers that can be checked by hand."""
    import torch

    import i8_ref as ref
    codes, s = ref.quantize(torch.tensor([[127.0, 0.5, 1.5, -2.5, 0.0], [0.0] * 5,
                                          [1.0, float("nan"), 0, 0, 0]], dtype=torch.float64))
    assert codes.tolist() == [[127, 0, 2, -2, 0], [0] * 5, [0] * 5]
    assert s[:2].tolist() == [1.0, 0.0] and s[2].isnan()
    out = ref.product(codes[:1], s[:1], codes[:1], s[:1] * 0.5, torch.float32)
    assert out.tolist() == [[(127 ** 2 + 8) * 0.5]]
    logp, stats, _ = ref.score(torch.log(torch.tensor([[1.0, 1, 2], [0, 0, 0], [1, 0, 0]],
                                                      dtype=torch.float64)),
                               torch.tensor([0, 1, 0]), 1.0)
    want = 0.5 * torch.log(torch.tensor(4.0, dtype=torch.float64)) + 0.5 * torch.log(torch.tensor(2.0))
    assert abs(float(logp[0] + torch.log(torch.tensor(4.0)))) < 1e-6
    assert abs(float(stats[0, 2] - want)) < 1e-6
    assert stats[1].tolist() == [float("-inf"), float("-inf"), 0.0] and logp[1] == float("-inf")
    assert logp[2] == 0 and stats[2, 2] == 0
