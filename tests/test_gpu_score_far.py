"""Log probabilities where two logits are further apart than binary32's largest number, and a
temperature of their size makes their probabilities alike."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _rows(torch, vocab, dtype):
    """The ends of the type among others: in the first vector, far behind it, at the row's end, the
    larger one first and last, with masked columns and without."""
    dt = getattr(torch, dtype)
    most = torch.finfo(dt).max
    z = torch.randn((8, vocab), generator=torch.Generator().manual_seed(1)) * 2.0 ** 126
    z = z.clamp(-2.0 ** 127, 2.0 ** 127)
    z[0, 0], z[0, -1] = most, -most
    z[1, 0], z[1, -1] = -most, most
    z[2, 3], z[2, 4] = -most, most
    z[3] = -most
    z[3, -2] = most
    z[4, ::2] = -most
    z[4, 1] = most
    z[5, 2:] = -torch.inf
    z[5, 0], z[5, 1] = -most, most
    z[6, :-1] = -most
    z[6, -1] = 2.0 ** 127
    z[7, 0], z[7, 1], z[7, 2] = most, -most, -torch.inf
    tokens = torch.tensor([vocab - 1, 0, 3, 5, 2, 0, 1, 2], dtype=torch.int32, device="cuda")
    return z.to(dt).cuda(), tokens


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab", [11, 3001, 20003])
@pytest.mark.parametrize("tau", [2.0 ** 124, 1e38, 3.4e38, 2.0 ** 100, 1.0])
def test_distances_past_binary32(torch, dtype, vocab, tau):
    """A distance is finite wherever it is so over tau.  Bounds: tests/score_ref.py; a log
    probability's own distance is a difference and a division, 4 U of it."""
    import i8_ref
    import paper_2202_06009_amd as zo
    import score_ref as ref
    z, tokens = _rows(torch, vocab, dtype)
    tau = float(torch.tensor(tau))
    logp, stats = torch.empty(8, device="cuda"), torch.empty((8, 3), device="cuda")
    values = torch.empty((8, 9), device="cuda")
    columns = torch.empty((8, 9), dtype=torch.int32, device="cuda")
    zo.zo_token_logprobs(z, tokens, logp, stats, values, columns, tau=tau)
    z64 = z.double()
    want, want_stats = ref.score(z64, tokens, tau)
    log_off, h_off = ref.off(z64, tau, 16 // z.element_size(), apart=True)
    assert torch.equal(stats[:, 0].double(), want_stats[:, 0])
    assert bool(((stats[:, 1] - want_stats[:, 1]).abs() <= log_off).all())
    assert bool(((stats[:, 2] - want_stats[:, 2]).abs() <= h_off).all())

    def near(got, z, stats, log_off):
        want = (z - stats[..., 0]) / tau - stats[..., 1]
        far = want < -torch.finfo(torch.float32).max          # as it rounds
        off = log_off + 5 * ref.U * (want.abs() + stats[..., 1])
        ok = torch.where(far, got == -torch.inf, (got - want).abs() <= off)
        assert bool(ok.all()), (got[~ok], want[~ok])

    near(logp.double(), z64.gather(1, tokens.long()[:, None])[:, 0], want_stats, log_off)
    at = columns.long()
    near(values.double(), z64.gather(1, at), want_stats[:, None], log_off[:, None])
    # the gradient, from exact statistics
    dlogp = torch.tensor([1.0, -2, 3, 1, 0, 1, -1, 2], device="cuda") * tau
    dentropy = torch.tensor([0.5, 0, 1, -1, 1, 0.25, 1, 0], device="cuda") * tau
    if tau * 4 < torch.finfo(torch.float32).max:
        dz = torch.empty_like(z)
        zo.zo_token_logprobs_grad(z, want_stats.float(), dz, tokens=tokens, dlogp=dlogp,
                                  dentropy=dentropy, tau=tau)
        want, off = i8_ref.score_grad(z64, tokens, tau, want_stats, dlogp, dentropy)
        half, tiny = i8_ref.HALF[z.dtype], i8_ref.TINY[z.dtype]
        assert bool(((dz.double() - want).abs() <= off + half * (want.abs() + off) + tiny).all())
