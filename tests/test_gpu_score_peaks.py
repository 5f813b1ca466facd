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


@pytest.mark.parametrize("dtype,vocab", CASES + [("float32", 9), ("bfloat16", 1003), ("float32", 140001)])
def test_confident_rows_keep_their_digits(torch, dtype, vocab):
    """log S = log1p(S - 1) where the largest logit has more than half of the row's probability,
    S - 1 summed apart from its 1: log probabilities and entropies down to 1e-18 are right in
    relation to themselves."""
    import score_ref as ref
    for tau in (1.0, 0.7):
        z, at = _peaked(torch, vocab, dtype, [2 + 0.7 * i for i in range(64)], seed=vocab + 1)
        at = z.argmax(1).int()
        logp, stats, _, _ = _score(torch, z, at, 3, tau)
        t = float(torch.tensor(tau))
        want, want_stats = ref.score(z.double(), at, t)
        log_off, h_off = ref.off(z.double(), t, _vec(z), apart=True)
        log_err, h_err = (stats[:, 1:].double() - want_stats[:, 1:]).abs().unbind(1)
        print("log S %.2f, entropy %.2f of the bound, log S from %.1e, bounds up to %.1e of it" % (
            float((log_err / log_off).max()), float((h_err / h_off).max()),
            float(want_stats[:, 1].min()), float((log_off / want_stats[:, 1]).max())))
        assert bool((log_err <= log_off).all()) and bool((h_err <= h_off).all())
        # the largest logit's log probability is the same number but for its sign
        assert torch.equal(logp, -stats[:, 1])


def test_equal_largest_logits(torch):
    """Two or more of them, in one vector, one lane, two lanes, among the last columns: each counts."""
    import score_ref as ref
    vocab = 20003
    for dtype in DTYPES:
        z = torch.randn((8, vocab), generator=torch.Generator().manual_seed(1)).to(getattr(torch, dtype))
        turn = 1024 * _vec(z)
        for i, cols in enumerate(([5], [5, 6], [5, 5 + turn], [5, 900], [vocab - 1], [vocab - 1, 7],
                                  [vocab - 1, vocab - 2], list(range(100)))):
            z[i, cols] = 30.0
        z = z.cuda()
        at = torch.tensor([5, 6, 5, 900, vocab - 1, 7, vocab - 2, 99], dtype=torch.int32, device="cuda")
        _, stats, values, columns = _score(torch, z, at, 2, 1.0)
        want = ref.score(z.double(), at, 1.0)[1]
        log_off, h_off = ref.off(z.double(), 1.0, _vec(z), apart=True)
        assert bool(((stats[:, 1] - want[:, 1]).abs() <= log_off).all())
        assert bool(((stats[:, 2] - want[:, 2]).abs() <= h_off).all())


@pytest.mark.parametrize("dtype,vocab", [("float32", 9), ("float32", 8195), ("bfloat16", 50304)])
def test_gradient_of_confident_tokens(torch, dtype, vocab):
    """dz of the token, dlogp (1 - p) - dentropy p (log p + entropy), from the statistics of the
    forward pass, in relation to itself.  1 - p is off by as much as log p and by expm1's two steps;
    p (log p + entropy) by both statistics; each of five operations more by U, 8 U with p's
    exponential."""
    import i8_ref
    import paper_2202_06009_amd as zo
    import score_ref as ref
    z, _ = _peaked(torch, vocab, dtype, [3 + 0.6 * i for i in range(64)], seed=5)
    at = z.argmax(1).int()
    _, stats, _, _ = _score(torch, z, at, 3, 1.0)
    want_logp, want = ref.score(z.double(), at, 1.0)
    log_off, h_off = ref.off(z.double(), 1.0, _vec(z), apart=True)
    one = torch.ones(64, device="cuda")
    for dlogp, dentropy in ((one, None), (None, one), (one, -0.25 * one)):
        dz = torch.empty_like(z)
        zo.zo_token_logprobs_grad(z, stats, dz, tokens=at, dlogp=dlogp, dentropy=dentropy)
        got = dz.gather(1, at.long()[:, None])[:, 0].double()
        a = 0.0 if dlogp is None else 1.0
        b = 0.0 if dentropy is None else float(dentropy[0])
        p, h = want_logp.exp(), want[:, 2]
        first, second = -a * torch.expm1(want_logp), -b * p * (want_logp + h)
        off = a * (log_off + 5 * ref.U * want_logp.abs())
        off += abs(b) * (log_off + h_off + 8 * ref.U * (want_logp.abs() + h))
        off += 8 * ref.U * (first.abs() + second.abs())
        dt = z.dtype
        off = off + i8_ref.HALF[dt] * ((first + second).abs() + off) + i8_ref.TINY[dt]
        err = (got - first - second).abs()
        print("%.2f of the bound" % float((err / off).max()))
        assert bool((err <= off).all())


@pytest.mark.parametrize("dtype,vocab", [("bfloat16", 8000), ("bfloat16", 50304), ("float32", 20001)])
def test_confident_rows_in_any_batch(torch, dtype, vocab):
    """The same bits from the forms for short rows, few rows, many rows and many alternatives."""
    z, _ = _peaked(torch, vocab, dtype, [5 + 0.05 * i for i in range(700)], seed=9)
    at = z.argmax(1).int()
    many = _score(torch, z, at, 20, 1.0)
    for rows, top in ((3, 20), (500, 300), (700, 300), (700, 1)):
        got = _score(torch, z[-rows:], at[-rows:], top, 1.0)
        assert torch.equal(got[0], many[0][-rows:]) and torch.equal(got[1], many[1][-rows:])
        n = min(top, 20)
        assert torch.equal(got[2][:, :n], many[2][-rows:, :n])
        assert torch.equal(got[3][:, :n], many[3][-rows:, :n])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [20003, 70001])
def test_masked_confident_rows(torch, dtype, vocab):
    """Masks of -infinity and of a low value before, around and behind the largest logit: the first
    1024 vectors altogether, all but it, all but it and one more, every second; rows that grow
    with every vector; a NaN beside them."""
    import score_ref as ref
    dt = getattr(torch, dtype)
    z = torch.randn((10, vocab), generator=torch.Generator().manual_seed(2)) * 2
    span = 1024 * (16 // torch.empty(0, dtype=dt).element_size())
    low = float(torch.finfo(dt).min)
    z[0, :span], z[0, span + 9] = -torch.inf, 25.0
    z[1, :], z[1, -1] = -torch.inf, 3.0
    z[2, :], z[2, -2], z[2, 17] = -torch.inf, 3.0, -20.0
    z[3, ::2], z[3, span + 1] = -torch.inf, 30.0
    z[4, :span], z[4, span + 9] = low, 25.0
    z[5, :], z[5, 5], z[5, -1] = low, 2.0, 14.0
    z[6] = torch.arange(vocab) // (span // 8) * 3.0
    z[6, -1] = float(z[6, -1]) + 20.0
    z[7] = -torch.arange(vocab) // (span // 8) * 3.0
    z[7, 0] = 20.0
    z[8, 3], z[9, 4], z[9, vocab // 2] = torch.nan, 30.0, low
    z = z.to(dt).cuda()
    fine = [0, 1, 2, 3, 4, 5, 6, 7, 9]
    at = z.nan_to_num(0.0, posinf=0.0, neginf=low).argmax(1).int()
    logp, stats, values, columns = _score(torch, z, at, 2, 1.0)
    assert bool(stats[8].isnan().all()) and bool(logp[8].isnan())
    want_logp, want = ref.score(z[fine].double(), at[fine], 1.0)
    log_off, h_off = ref.off(z[fine].double(), 1.0, 16 // z.element_size(), apart=True)
    err = (stats[fine].double() - want).abs()
    assert not bool(err[:, 0].any()) and torch.equal(columns[fine, 0], at[fine])
    assert bool((err[:, 1] <= log_off).all()), (err[:, 1], log_off)
    assert bool((err[:, 2] <= h_off).all()), (err[:, 2], h_off)
    assert bool(((logp[fine].double() - want_logp).abs() <= log_off).all())
    assert torch.equal(values[fine, 0], logp[fine])
