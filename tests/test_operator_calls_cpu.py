"""The operators' binding and host checks beyond test_operators_cpu.py: no kernel is
launched."""
import ctypes
import types

import pytest

import paper_2202_06009_amd as zo
from paper_2202_06009_amd import operators


def test_stream_of_another_gpu_is_refused(monkeypatch):
    """Every GPU's default stream has the handle 0, so the handle alone tells nothing."""
    called = []
    monkeypatch.setitem(operators._functions, "zo_mx4_product",
                        lambda *a: called.append(a) or zo.ZO_OK)
    monkeypatch.setattr(operators.torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(operators.torch._C, "_cuda_getCurrentRawStream", lambda dev: 0,
                        raising=False)
    with pytest.raises(ValueError):
        operators._run("zo_mx4_product", 0, types.SimpleNamespace(device_index=1, cuda_stream=0),
                       (), ())
    assert not called
    operators._run("zo_mx4_product", 0, types.SimpleNamespace(device_index=0, cuda_stream=0),
                   (), ())
    assert len(called) == 1


P = 1 << 20        # stands for a device pointer in calls that are refused


def test_matrices_beyond_a_launch_are_refused():
    """2^24 workgroups of 256 threads, 2^23 of 512: one more than a launch holds."""
    L = zo.lib()
    most = 1 << 30

    def at(rows, cols):
        return ctypes.byref(zo._Mx4(P, P, rows, cols))
    assert L.zo_mx4_quantize(P, 0, most, 1, 1, at(most, 1), None, None) == zo.ZO_EINVAL
    assert L.zo_mx4_quantize(P, 1, most, 129, 129, at(most, 129), None, None) == zo.ZO_EINVAL
    assert L.zo_mx4_quantize(P, 2, 200, most, most, None, at(most, 200), None) == zo.ZO_EINVAL
    assert L.zo_mx4_dequantize(at(most, 5), P, 2, 5, None) == zo.ZO_EINVAL
    assert L.zo_mx4_product(at(1, 10), at(most, 10), P, 2, most, None) == zo.ZO_EINVAL
    assert L.zo_mx4_product(at(300, 10), at(most, 10), P, 2, most, None) == zo.ZO_EINVAL
    assert L.zo_mx4_linear(P, 2, 10, at(most, 10), at(1, 10), P, 2, most, None) == zo.ZO_EINVAL
    # the activations' quantisation, before anything is launched
    assert L.zo_mx4_linear(P, 0, 1, at(1, 1), at(most, 1), P, 2, 1, None) == zo.ZO_EINVAL
