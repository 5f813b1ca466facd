"""Log probabilities and entropies of confident rows: one logit far above the others, wherever it
stands in the row."""
import pytest

pytestmark = pytest.mark.gpu

DTYPES = ["float32", "float16", "bfloat16"]


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _vec(z):
    return 16 // z.element_size()


def _peaked(torch, vocab, dtype, peaks, seed=0):
    """A bulk and one logit above it in every row: in a lane's first vector, a later one, the last
    whole one, among the columns behind it.  Returns z, the columns."""
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((len(peaks), vocab), generator=g) * 2.0
    at = torch.randint(0, vocab, (len(peaks),), generator=g)
    at[::5] = vocab - 1
    at[1::5] = torch.clamp(at[1::5], min=vocab // 2)
    rows = torch.arange(len(peaks))
    z[rows, at] = torch.as_tensor(peaks, dtype=torch.float32) + torch.rand(len(peaks), generator=g)
    return z.to(getattr(torch, dtype)).cuda(), at.int().cuda()


def _score(torch, z, tokens, top, tau):
    import paper_2202_06009_amd as zo
    rows = len(z)
    logp, stats = torch.empty(rows, device="cuda"), torch.empty((rows, 3), device="cuda")
    values = torch.empty((rows, top), device="cuda")
    columns = torch.empty((rows, top), dtype=torch.int32, device="cuda")
    zo.zo_token_logprobs(z, tokens, logp, stats, values, columns, tau=tau)
    return logp, stats, values, columns


CASES = [("float32", 8192), ("float32", 8195), ("float32", 50257), ("float16", 16389),
         ("bfloat16", 16384), ("bfloat16", 50304), ("bfloat16", 9000)]


@pytest.mark.parametrize("dtype,vocab", CASES)
def test_no_log_probability_above_0(torch, dtype, vocab):
    """exp(logp) stays a probability, log S is not below 0 and the gradient of the token's own
    logit does not turn round, for few rows and for many."""
    import paper_2202_06009_amd as zo
    for tau in (1.0, 0.7):
        for rows in (60, 600):
            z, at = _peaked(torch, vocab, dtype, [8 + 36 * i / rows for i in range(rows)], seed=rows)
            logp, stats, values, _ = _score(torch, z, at, 3, tau)
            assert bool((stats[:, 1] >= 0).all()), float(stats[:, 1].min())
            assert bool((stats[:, 2] >= 0).all()), float(stats[:, 2].min())
            assert bool((logp <= 0).all()) and bool((values <= 0).all()), float(logp.max())
            dz = torch.empty_like(z)
            zo.zo_token_logprobs_grad(z, stats, dz, tokens=at, dlogp=torch.ones(rows, device="cuda"),
                                      tau=tau)
            own = dz.gather(1, at.long()[:, None])
            assert bool((own >= 0).all())


@pytest.mark.parametrize("dtype,vocab", CASES)
def test_entropy_of_peaked_rows(torch, dtype, vocab):
    """Sums about logits that are at least as large as their terms' have no parts that cancel."""
    import score_ref as ref
    for tau in (1.0, 0.7):
        z, at = _peaked(torch, vocab, dtype, [4 + 0.6 * i for i in range(64)], seed=vocab)
        logp, stats, _, _ = _score(torch, z, at, 3, tau)
        tau = float(torch.tensor(tau))
        want, want_stats = ref.score(z.double(), at, tau)
        log_off, h_off = ref.off(z.double(), tau, _vec(z), apart=False)
        d = (stats[:, 0].double() - z.double().gather(1, at.long()[:, None])[:, 0]) / tau
        print("log S %.2f, entropy %.2f of the bound" % (
            float(((stats[:, 1] - want_stats[:, 1]).abs() / log_off).max()),
            float(((stats[:, 2] - want_stats[:, 2]).abs() / h_off).max())))
        assert torch.equal(stats[:, 0].double(), want_stats[:, 0])
        assert bool(((stats[:, 1] - want_stats[:, 1]).abs() <= log_off).all())
        assert bool(((stats[:, 2] - want_stats[:, 2]).abs() <= h_off).all())
        assert bool(((logp - want).abs() <= log_off + 4 * ref.U * d + ref.U * want.abs()).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_entropy_of_few_logits(torch, dtype):
    """A lane's first vector holds one small logit, its next one the row's largest, and the row
    four more: an addition of 0 is none, so seven additions and three moves of a sum by 3 U each
    are all that is rounded beside the terms themselves."""
    import score_ref as ref
    g = torch.Generator().manual_seed(3)
    for many in (False, True):                          # both forms of long rows
        rows = 640 if many else 64
        z = torch.full((rows, 20000), -torch.inf, dtype=getattr(torch, dtype))
        turn = 1024 * _vec(z)
        for i in range(rows):
            peak = 10.0 + 34.0 * i / rows
            lane = int(torch.randint(0, 20000 - turn, (1,), generator=g))
            others = torch.randint(0, 20000, (4,), generator=g)
            z[i, others] = (torch.rand(4, generator=g) * (peak - 3)).to(z.dtype)
            z[i, lane], z[i, lane + turn] = 0.125, peak
        z = z.cuda()
        at = z.argmax(1).int()
        _, stats, _, _ = _score(torch, z, at, 3, 1.0)
        want = ref.score(z.double(), at, 1.0)[1]
        log_off, h_off = ref.off(z.double(), 1.0, _vec(z), apart=False, count=7 + 9)
        print("log S %.2f, entropy %.2f of the bound" % (
            float(((stats[:, 1] - want[:, 1]).abs() / log_off).max()),
            float(((stats[:, 2] - want[:, 2]).abs() / h_off).max())))
        assert bool(((stats[:, 1] - want[:, 1]).abs() <= log_off).all())
        assert bool(((stats[:, 2] - want[:, 2]).abs() <= h_off).all())
