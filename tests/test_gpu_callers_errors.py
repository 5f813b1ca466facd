"""An error that the caller's own HIP call left behind is not the operators': a call that
launches its kernels returns ZO_OK, and the error is there for the caller afterwards."""
import pytest

pytestmark = pytest.mark.gpu


def test_an_earlier_error_is_not_reported():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2202_06009_amd as zo
    x = torch.randn((70, 200), device="cuda")
    w = torch.randn((300, 200), device="cuda")
    big = torch.randn((4200, 1100), device="cuda")
    xq, wq, bq = zo.Mx4(70, 200), zo.Mx4(300, 200), zo.Mx4(4200, 1100)
    few, y, back = (torch.empty(s, device="cuda") for s in ((70, 300), (70, 300), (300, 200)))
    yb = torch.empty((4200, 4200), dtype=torch.bfloat16, device="cuda")
    values = torch.empty((70, 4), device="cuda")
    columns = torch.empty((70, 4), dtype=torch.int32, device="cuda")
    loss = torch.empty(70, device="cuda")
    torch.cuda.synchronize()
    hip = zo.lib()                               # the runtime that the library is linked to
    calls = [lambda: zo.zo_mx4_quantize(x, xq), lambda: zo.zo_mx4_quantize(w, wq),
             lambda: zo.zo_mx4_quantize(big, bq), lambda: zo.zo_mx4_dequantize(wq, back),
             lambda: zo.zo_mx4_product(xq, wq, y), lambda: zo.zo_mx4_product(bq, bq, yb),
             lambda: zo.zo_mx4_linear(x[:3], wq, few[:3], zo.Mx4(3, 200)),
             lambda: zo.zo_top_logits(x, values, columns),
             lambda: zo.zo_top_logits(x, values, columns, loss),
             lambda: zo.zo_distill_loss(x, values, columns, loss)]
    try:
        for call in calls:
            assert hip.hipSetDevice(1 << 20) != 0
            call()
            assert hip.hipGetLastError() != 0
    finally:
        hip.hipGetLastError()
    torch.cuda.synchronize()
    assert torch.isfinite(y).all() and torch.isfinite(loss).all()
