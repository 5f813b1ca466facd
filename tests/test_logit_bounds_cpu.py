"""The limits of logit_bounds.py reject a result that is wrong, in every row: the oracle's
own, moved a little, stands in for a kernel's."""
import numpy as np
import pytest

import logit_bounds as lb
import operators_ref as ref

LOWEST = {"float32": -lb.FLT_MAX, "float16": -65504.0, "bfloat16": -float.fromhex("0x1.fep127")}


@pytest.mark.parametrize("tail", [False, True])
def test_agrees_with_the_oracle(tail):
    """The definition written a second time, on rows that need no care."""
    r = np.random.default_rng(4)
    z = r.normal(size=(30, 90)) * 3
    z[3, 5:9] = -np.inf
    vals, cols, lse = lb._nearby_teacher(r, z, 7, 1.5)
    cols[2, 3:], cols[4] = -1, [1, 1, 2, 3, 2, 90, -1]
    labels = r.integers(-1, 91, 30)
    kw = dict(tau=1.5, lse=lse if tail else None, labels=labels, kd=0.7, ce=0.4,
              weight=r.normal(size=30))
    want, want_dz = ref.distill(z, vals.astype(np.float64), cols, **kw)
    loss, dz, lim, lim_dz = lb.distill(z, vals, cols, "float32", **kw)
    np.testing.assert_allclose(loss, want, rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(dz, want_dz, rtol=1e-12, atol=1e-12)
    assert lim.max() < 1e-3 and lim_dz.max() < 1e-4


def _rejects(case, dtype, kw, skip=()):
    z, vals, cols = case[:3]
    with np.errstate(all="ignore"):
        loss, dz, lim_loss, lim_dz = lb.distill(z, vals, cols, dtype, **kw)
    weight = kw.get("weight")
    for t in range(len(z)):
        if t in skip or (weight is not None and weight[t] == 0):
            continue
        assert np.isfinite(lim_loss[t]) and np.isfinite(lim_dz[t]).all(), t
        if np.isfinite(loss[t]):
            assert lim_loss[t] <= 0.04 * max(1.0, abs(loss[t])), (t, loss[t], lim_loss[t])
        i = np.argmax(np.abs(dz[t]))
        if dz[t, i] != 0:
            part = 0.02 if dtype == "bfloat16" else 0.01
            assert lim_dz[t, i] <= part * abs(dz[t, i]) + 1e-5, (t, dz[t, i], lim_dz[t, i])


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0])
def test_far_rest(dtype, tau):
    case = lb.far_rest_rows(700, tau, [-100.0, -1e4, max(-1e9, LOWEST[dtype]), LOWEST[dtype]], True)
    _rejects(case, dtype, dict(tau=tau, lse=case[3], labels=case[4], kd=0.7, ce=0.3))
    _rejects(case, dtype, dict(tau=tau, lse=case[3]))


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("tau", [1.0, 2.0, 1.5])
def test_masked(tau, tail):
    case = lb.masked_rows(700, tau, LOWEST["float32"])
    _rejects(case, "float32", dict(tau=tau, lse=case[3] if tail else None, labels=case[4], ce=0.5,
                                   weight=case[5]))


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("tau", [1.0, 2.0, 1.5])
def test_extreme(tau, tail):
    case = lb.extreme_rows(700, tau)
    _rejects(case, "float32", dict(tau=tau, lse=case[3] if tail else None, labels=case[4], ce=0.5))


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("tau", [1.0, 2.0, 1.5])
def test_large(tau, tail):
    case = lb.large_rows(700, tau)
    _rejects(case, "float32", dict(tau=tau, lse=case[3] if tail else None, labels=case[4], ce=0.5))
