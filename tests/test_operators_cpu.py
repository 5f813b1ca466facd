"""The operators' refusals, sizes and oracle on the CPU: no kernel is launched."""
import ctypes

import numpy as np
import pytest

import operators_ref as ref
import paper_2202_06009_amd as zo

P = 1 << 20        # stands for a device pointer in calls that are refused


def _mx4(rows, cols, codes=P, scales=P):
    return zo._Mx4(codes, scales, rows, cols)


def test_mx4_sizes():
    assert zo.zo_mx4_code_bytes(0, 5) == 0 and zo.zo_mx4_scale_bytes(5, 0) == 0
    assert zo.zo_mx4_code_bytes(1, 1) == 64 * 64 and zo.zo_mx4_scale_bytes(1, 1) == 64 * 4
    assert zo.zo_mx4_code_bytes(65, 1600) == 128 * 13 * 64
    assert zo.zo_mx4_scale_bytes(65, 1600) == 128 * 13 * 4
    # past 32 bits
    assert zo.zo_mx4_code_bytes(1 << 20, 1 << 16) == 1 << 35
    for bad in ((-1, 1), (1, -1), ((1 << 30) + 1, 1)):
        for f in (zo.zo_mx4_code_bytes, zo.zo_mx4_scale_bytes):
            with pytest.raises(zo.ZoError) as e:
                f(*bad)
            assert e.value.status == zo.ZO_EINVAL


@pytest.mark.parametrize("over,code", [
    (dict(dtype=3), zo.ZO_EINVAL), (dict(dtype=-1), zo.ZO_EINVAL),
    (dict(x=None), zo.ZO_EINVAL), (dict(rows=-1), zo.ZO_EINVAL), (dict(ld=9), zo.ZO_EINVAL),
    (dict(x=P + 2), zo.ZO_EALIGN), (dict(dtype=1, x=P + 1), zo.ZO_EALIGN),
    (dict(q=None), zo.ZO_EINVAL), (dict(q=_mx4(4, 11)), zo.ZO_EINVAL),
    (dict(qt=_mx4(4, 10)), zo.ZO_EINVAL), (dict(q=_mx4(4, 10, codes=None)), zo.ZO_EINVAL),
    (dict(q=_mx4(4, 10, codes=P + 8)), zo.ZO_EALIGN),
    (dict(q=_mx4(4, 10, scales=P + 2)), zo.ZO_EALIGN),
    (dict(rows=0, q=_mx4(0, 10), x=None), zo.ZO_OK),
])
def test_quantize_refusals(over, code):
    a = dict(x=P, dtype=0, rows=4, cols=10, ld=10, q=_mx4(4, 10), qt=None)
    a.update(over)
    at = [ctypes.addressof(m) if m is not None else None for m in (a["q"], a["qt"])]
    assert zo.lib().zo_mx4_quantize(a["x"], a["dtype"], a["rows"], a["cols"], a["ld"], *at,
                                    None) == code


def test_quantize_refuses_both_outputs_missing():
    assert zo.lib().zo_mx4_quantize(P, 0, 4, 10, 10, None, None, None) == zo.ZO_EINVAL


@pytest.mark.parametrize("a,b,out,dtype,ld,code", [
    (_mx4(4, 10), _mx4(5, 11), P, 0, 5, zo.ZO_EINVAL),       # reduced axes differ
    (_mx4(4, 10), _mx4(5, 10), None, 0, 5, zo.ZO_EINVAL),
    (_mx4(4, 10), _mx4(5, 10), P, 7, 5, zo.ZO_EINVAL),
    (_mx4(4, 10), _mx4(5, 10), P, 0, 4, zo.ZO_EINVAL),
    (_mx4(4, 10), _mx4(5, 10), P + 1, 2, 5, zo.ZO_EALIGN),
    (_mx4(4, 10, codes=None), _mx4(5, 10), P, 0, 5, zo.ZO_EINVAL),
    (_mx4(4, 10), _mx4(5, 10, codes=P + 4), P, 0, 5, zo.ZO_EALIGN),
    (_mx4(1 << 30, 10), _mx4(1 << 30, 10), P, 0, 1 << 30, zo.ZO_EINVAL),   # one launch's grid
    (_mx4(0, 10, codes=None), _mx4(5, 10), None, 0, 5, zo.ZO_OK),
])
def test_product_and_linear_refusals(a, b, out, dtype, ld, code):
    ra, rb = ctypes.byref(a), ctypes.byref(b)
    L = zo.lib()
    assert L.zo_mx4_product(ra, rb, out, dtype, ld, None) == code
    if a.rows:
        assert L.zo_mx4_linear(P, 2, 10, rb, ra, out, dtype, ld, None) == code
    assert L.zo_mx4_product(None, rb, P, 0, 5, None) == zo.ZO_EINVAL


def test_linear_and_dequantize_refusals():
    L = zo.lib()
    w, xq = _mx4(5, 10), _mx4(4, 10)
    assert L.zo_mx4_linear(None, 2, 10, ctypes.byref(w), ctypes.byref(xq), P, 0, 5,
                           None) == zo.ZO_EINVAL
    assert L.zo_mx4_linear(P, 2, 9, ctypes.byref(w), ctypes.byref(xq), P, 0, 5,
                           None) == zo.ZO_EINVAL
    assert L.zo_mx4_linear(P + 1, 2, 10, ctypes.byref(w), ctypes.byref(xq), P, 0, 5,
                           None) == zo.ZO_EALIGN
    assert L.zo_mx4_dequantize(None, P, 0, 10, None) == zo.ZO_EINVAL
    assert L.zo_mx4_dequantize(ctypes.byref(w), P, 0, 9, None) == zo.ZO_EINVAL
    assert L.zo_mx4_dequantize(ctypes.byref(w), P + 2, 0, 10, None) == zo.ZO_EALIGN


@pytest.mark.parametrize("over,code", [
    (dict(top=0), zo.ZO_EINVAL), (dict(top=101), zo.ZO_EINVAL),
    (dict(top=1025, vocab=2000, ld=2000), zo.ZO_EINVAL), (dict(vocab=0), zo.ZO_EINVAL),
    (dict(vocab=1 << 31, ld=1 << 31), zo.ZO_EINVAL), (dict(rows=-1), zo.ZO_EINVAL),
    (dict(tau=0.0), zo.ZO_EINVAL), (dict(tau=float("nan")), zo.ZO_EINVAL),
    (dict(tau=float("inf")), zo.ZO_EINVAL), (dict(ld=99), zo.ZO_EINVAL),
    (dict(dtype=5), zo.ZO_EINVAL), (dict(z=None), zo.ZO_EINVAL),
    (dict(values=None), zo.ZO_EINVAL), (dict(columns=None), zo.ZO_EINVAL),
    (dict(z=P + 2), zo.ZO_EALIGN), (dict(lse=P + 1), zo.ZO_EALIGN),
    (dict(rows=0, z=None, values=None), zo.ZO_OK),
])
def test_top_logits_refusals(over, code):
    a = dict(z=P, dtype=0, rows=3, vocab=100, ld=100, top=7, tau=1.0, values=P, columns=P, lse=P)
    a.update(over)
    assert zo.lib().zo_top_logits(*a.values(), None) == code


def _distill(**over):
    a = dict(z=P, dtype=2, rows=3, vocab=100, ldz=100, top=7, values=P, columns=P,
             teacher_lse=None, labels=None, row_weight=None, tau=1.0, kd_weight=1.0,
             ce_weight=0.0, loss=P, dz=2 * P, lddz=100)
    a.update(over)
    return zo._Distill(**a)


@pytest.mark.parametrize("over,code", [
    (dict(top=0), zo.ZO_EINVAL), (dict(top=1025), zo.ZO_EINVAL), (dict(vocab=0), zo.ZO_EINVAL),
    (dict(vocab=(1 << 18) + 1, ldz=1 << 19, lddz=1 << 19), zo.ZO_EINVAL),
    (dict(rows=-1), zo.ZO_EINVAL), (dict(dtype=9), zo.ZO_EINVAL), (dict(z=None), zo.ZO_EINVAL),
    (dict(ldz=99), zo.ZO_EINVAL), (dict(lddz=99), zo.ZO_EINVAL), (dict(values=None), zo.ZO_EINVAL),
    (dict(columns=None), zo.ZO_EINVAL), (dict(loss=None, dz=None), zo.ZO_EINVAL),
    (dict(dz=P, lddz=104), zo.ZO_EINVAL),                      # in place with another stride
    (dict(tau=-1.0), zo.ZO_EINVAL), (dict(kd_weight=float("nan")), zo.ZO_EINVAL),
    (dict(ce_weight=float("inf")), zo.ZO_EINVAL), (dict(z=P + 1), zo.ZO_EALIGN),
    (dict(dz=2 * P + 1), zo.ZO_EALIGN), (dict(labels=P + 2), zo.ZO_EALIGN),
    (dict(row_weight=P + 2), zo.ZO_EALIGN), (dict(teacher_lse=P + 2), zo.ZO_EALIGN),
    (dict(rows=0, z=None), zo.ZO_OK),
])
def test_distill_refusals(over, code):
    assert zo.lib().zo_distill_loss(ctypes.byref(_distill(**over)), None) == code
    assert zo.lib().zo_distill_loss(None, None) == zo.ZO_EINVAL


def test_wrapper_refuses_host_tensors():
    import torch
    with pytest.raises(ValueError):
        zo.zo_mx4_quantize(torch.zeros(2, 2))
    with pytest.raises(ValueError):
        zo.zo_top_logits(torch.zeros(2, 9), torch.zeros(2, 1), torch.zeros(2, 1, dtype=torch.int32))
    with pytest.raises(ValueError):
        zo.Mx4(4, 4, codes=torch.zeros(3, dtype=torch.uint8))
    with pytest.raises(ValueError):
        zo.Mx4(4, 4, codes=torch.zeros(1 << 14))


# --------------------------------------------------------------- the oracle itself

def test_oracle_rounds_to_nearest_even():
    x = np.array([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9, -0.25, 0.2500001, -6.0, 4.0]])
    code, byte = ref.quantize(x)
    assert byte[0, 0] == 127
    np.testing.assert_array_equal(ref.GRID[code[0]], [0, 1, 1, 2, 2, 4, 4, 6, -0.0, 0.5, -6, 4])


def test_oracle_scales():
    for a, b in ((4.0, 127), (7.99, 127), (8.0, 128), (3.99, 126), (2.0 ** -125, 0),
                 (2.0 ** -149, 0), (0.0, 0), (2.0 ** 127, 252), (np.inf, 255), (np.nan, 255)):
        x = np.zeros((1, 32))
        x[0, 5] = a
        assert ref.quantize(x)[1][0, 0] == b, a


def test_oracle_distill_gradient_is_the_difference_quotient():
    r = np.random.default_rng(3)
    z = r.normal(size=(4, 19)) * 2
    cols = np.stack([r.permutation(19)[:5] for _ in range(4)]).astype(np.int32)
    cols[1, 2] = -1
    vals = np.take_along_axis(z, np.maximum(cols, 0), 1) + r.normal(size=(4, 5))
    lse = ref.log_sum_exp(np.concatenate([vals, z], 1) / 1.7)
    for kw in (dict(), dict(lse=lse), dict(lse=lse, labels=np.array([3, -1, 18, 0]), ce=0.4)):
        kw = dict(kw, tau=1.7, kd=0.6, weight=np.array([1.0, 0.5, 2.0, 0.0]))
        _, dz = ref.distill(z, vals, cols, **kw)
        h = 1e-5
        for i in range(19):
            up, dn = z.copy(), z.copy()
            up[:, i] += h
            dn[:, i] -= h
            num = (ref.distill(up, vals, cols, **kw)[0] - ref.distill(dn, vals, cols, **kw)[0])
            np.testing.assert_allclose(dz[:, i], num / (2 * h), atol=1e-8)
