"""The operators' binding and host checks beyond test_operators_cpu.py: no kernel is
launched."""
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
