"""Forms of the 4-bit kernels that a call's sizes, types and alignment choose: values read
back where rows begin on lines of 128 bytes, products of large tiles in binary16."""
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


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("shape", [(1, 1), (3, 33), (64, 128), (66, 129), (200, 320), (130, 1601),
                                   (65, 127), (257, 4095)])
def test_dequantize_on_lines(torch, shape, dtype):
    """Rows a whole number of lines apart, the last line partly the matrix's: exact, and
    what is beside the matrix untouched; the same one element off the lines."""
    import paper_2202_06009_amd as zo
    rows, cols = shape
    r = np.random.default_rng(rows + cols)
    x = r.normal(size=shape) * np.exp2(r.integers(-9, 9, size=(rows, 1)))
    x[0, cols // 2] = np.nan
    x = torch.from_numpy(x).to(getattr(torch, dtype)).cuda()
    q = zo.Mx4(rows, cols)
    zo.zo_mx4_quantize(x, q)
    want = ref.rounded(x.double().cpu().numpy())
    if dtype == "float16":
        want = want.astype(np.float16).astype(np.float64)
    wide = -(-cols // 64) * 64 + 64
    for off in (0, 1):
        full = torch.full((rows + 2, wide), 7.0, dtype=x.dtype, device="cuda")
        assert full.data_ptr() % 128 == 0
        out = full[1:rows + 1, off:off + cols]
        zo.zo_mx4_dequantize(q, out)
        np.testing.assert_array_equal(out.double().cpu().numpy(), want)
        assert (full[0] == 7).all() and (full[-1] == 7).all()
        assert (full[:, :off] == 7).all() and (full[:, off + cols:] == 7).all()


def _check_product(torch, m, n, k, pad, dtype):
    import paper_2202_06009_amd as zo
    g = torch.Generator(device="cuda").manual_seed(m + n)
    a = torch.randn((m, k), generator=g, device="cuda")
    b = torch.randn((n, k), generator=g, device="cuda")
    aq, bq = zo.Mx4(m, k), zo.Mx4(n, k)
    zo.zo_mx4_quantize(a, aq)
    zo.zo_mx4_quantize(b, bq)
    va, vb = torch.empty_like(a), torch.empty_like(b)
    zo.zo_mx4_dequantize(aq, va)
    zo.zo_mx4_dequantize(bq, vb)
    wide = n + pad if pad < 64 else -(-n // 64) * 64
    full = torch.full((m, wide), 7.0, dtype=getattr(torch, dtype), device="cuda")
    zo.zo_mx4_product(aq, bq, full[:, :n])
    va, vb = va.double(), vb.double()
    want = va @ vb.t().contiguous()
    acc = (k + 8) * 2.0 ** -23 * (va.abs() @ vb.abs().t().contiguous())
    off = (full[:, :n].double() - want).abs()
    tiny = 2.0 ** -25 if dtype == "float16" else 2.0 ** -134
    assert bool((off <= acc + HALF_ULP[dtype] * (want.abs() + acc) + tiny).all())
    assert (full[:, n:] == 7).all()


@pytest.mark.parametrize("m,n,k", [(4200, 4303, 1020), (2500, 7296, 1300), (2050, 8200, 1024),
                                   (6333, 1601, 1200), (2300, 7300, 200), (1000, 2000, 300),
                                   (300, 500, 700)])
@pytest.mark.parametrize("pad", [0, 1, 64])
def test_product_in_binary16(torch, m, n, k, pad):
    _check_product(torch, m, n, k, pad, "float16")


# tiles of 256 x 256: 221 of one round, 384 and 544 of several with a rest that is halved, 420
# with one that is not; steps around the least for each, odd and even
@pytest.mark.parametrize("m,n,k", [(3300, 4350, 1100), (3300, 4350, 1500), (6100, 4050, 2090),
                                   (6100, 4050, 4200), (8100, 4200, 2000), (8100, 4200, 1900),
                                   (5333, 5097, 2433), (5333, 5097, 4100)])
@pytest.mark.parametrize("pad", [0, 64])
@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_product_of_large_tiles(torch, m, n, k, pad, dtype):
    _check_product(torch, m, n, k, pad, dtype)


@pytest.mark.parametrize("m", [1, 7, 8, 11, 16])
@pytest.mark.parametrize("n,k", [(6400, 2560), (6400, 6400), (4096, 6400), (4113, 4000), (25600, 512),
                                 (517, 6656), (130, 6657)])
def test_linear_is_quantize_and_product(torch, m, n, k):
    """The one-kernel form and the two kernels, on both sides of where one gives way to the
    other: the same bits."""
    import paper_2202_06009_amd as zo
    x = torch.randn((m, k), device="cuda").bfloat16()
    w = zo.Mx4(n, k)
    zo.zo_mx4_quantize(torch.randn((n, k), device="cuda"), w)
    one, two = (torch.full((m, n), 7.0, device="cuda") for _ in range(2))
    xq = zo.Mx4(m, k)
    zo.zo_mx4_linear(x, w, one, zo.Mx4(m, k))
    zo.zo_mx4_quantize(x, xq)
    zo.zo_mx4_product(xq, w, two)
    assert torch.equal(one, two)
