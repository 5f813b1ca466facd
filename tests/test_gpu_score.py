"""Log probabilities, entropies, alternatives and their gradients on the GPU against the
64-bit oracle: orders bit for bit, the rest within what its roundings allow
(tests/i8_ref.py)."""
import pytest

pytestmark = pytest.mark.gpu

DTYPES = ["float32", "float16", "bfloat16"]
VOCABS = [1, 2, 7, 8, 9, 100, 1000, 1025, 2048, 2049, 8191, 16385, 30522, 50257, 50304]


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _logits(torch, rows, vocab, dtype, seed, pad=0, sigma=2.0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((rows, vocab), generator=g) * sigma
    z += 6.0 * (torch.rand((rows, vocab), generator=g) < 0.002)
    full = torch.full((rows, vocab + pad), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    full[:, :vocab] = z.to(full.dtype)
    return full[:, :vocab]


def _tokens(torch, z, seed):
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, z.shape[1], (len(z),), generator=g).cuda()
    t[::2] = z[::2].nan_to_num(-1e30).argmax(1)
    if len(z) > 3:
        t[1], t[3] = -1, z.shape[1]
    return t.int()


def _score(torch, z, tokens, top, tau=1.0, **kw):
    import paper_2202_06009_amd as zo
    rows = len(z)
    logp = torch.full((rows,), 7.0, device="cuda") if tokens is not None else None
    stats = torch.full((rows, 3), 7.0, device="cuda")
    values = torch.full((rows, top), 7.0, device="cuda") if top else None
    columns = torch.full((rows, top), -7, dtype=torch.int32, device="cuda") if top else None
    zo.zo_token_logprobs(z, tokens, logp, stats, values, columns, tau=tau, **kw)
    return logp, stats, values, columns


def _order(torch, z, top):
    """Columns by value, NaN before +infinity, the lowest first among equals."""
    key = torch.where(z.isnan(), torch.inf, z)
    at = torch.sort(key, dim=1, descending=True, stable=True).indices
    nan = torch.gather(z.isnan(), 1, at)
    return at.gather(1, torch.sort(nan.int(), dim=1, descending=True, stable=True).indices)[:, :top]


def _near(torch, got, want, off):
    want = torch.where(want < -torch.finfo(torch.float32).max, -torch.inf, want)   # as it rounds
    same = (got.double() == want) | (got.isnan() & want.isnan())
    bad = ~same & ~((got.double() - want).abs() <= off)
    assert not bool(bad.any()), (got[bad][:4], want[bad][:4])


def _check(torch, z, tokens, top, tau, got):
    import i8_ref as ref
    logp, stats, values, columns = got
    z64 = z.double()
    want, want_stats, all_logp = ref.score(z64, tokens, tau)
    log_off, h_off = ref.score_off(z64, tau)
    _near(torch, stats[:, 0], want_stats[:, 0], 0.0)
    _near(torch, stats[:, 1], want_stats[:, 1], log_off)
    _near(torch, stats[:, 2], want_stats[:, 2], h_off)
    # the distance of a logit from the largest: a subtraction and a division
    d = (all_logp + want_stats[:, 1:2]).abs().nan_to_num(0.0, posinf=0.0)
    if tokens is not None:
        has = (tokens >= 0) & (tokens < z.shape[1])
        at = torch.where(has, tokens, 0).long()[:, None]
        off = log_off + 4 * ref.U * d.gather(1, at)[:, 0] + ref.U * want.abs().nan_to_num(posinf=0)
        _near(torch, logp, want, off)
    if top:
        at = _order(torch, z64, top)
        assert torch.equal(columns.long(), at)
        want = all_logp.gather(1, at)
        _near(torch, values, want, log_off[:, None] + 4 * ref.U * d.gather(1, at) +
              ref.U * want.abs().nan_to_num(posinf=0))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_score(torch, vocab, dtype):
    for rows, pad, top, tau in ((1, 0, 1, 1.0), (5, 3, 20, 0.7), (9, 64, 300, 1.5), (4, 1, 0, 1.0)):
        z = _logits(torch, rows, vocab, dtype, seed=vocab + rows, pad=pad)
        tokens = _tokens(torch, z, seed=rows)
        top = min(top, vocab)
        _check(torch, z, tokens, top, tau, _score(torch, z, tokens, top, tau))


@pytest.mark.parametrize("dtype,vocab,top", [("float32", 70000, 5), ("bfloat16", 140000, 64),
                                             ("float16", 131073, 0), ("bfloat16", 131072, 1024),
                                             ("float32", 65537, 700)])
def test_score_long(torch, dtype, vocab, top):
    """Around and beyond what a workgroup's registers hold."""
    z = _logits(torch, 3, vocab, dtype, seed=1, pad=5)
    tokens = _tokens(torch, z, seed=2)
    _check(torch, z, tokens, top, 1.0, _score(torch, z, tokens, top))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [300, 50257, 140001])
def test_score_masks(torch, vocab, dtype):
    """Rows masked but for few columns, for one, altogether; by -infinity, by -1e4 and by the
    type's lowest value; equal logits throughout; NaN and +infinity; logits far out."""
    dt = getattr(torch, dtype)
    z = _logits(torch, 14, vocab, dtype, seed=4)
    low = torch.finfo(dt).min
    z[0, 40:] = -torch.inf
    z[1, :-1] = -torch.inf
    z[2] = -torch.inf
    z[3, 3:] = -1e4
    z[4, 7:] = low
    z[5] = 1.5
    z[6, vocab // 2] = torch.nan
    z[7, vocab // 3] = torch.inf
    z[8, 5], z[8, 6] = torch.nan, torch.inf
    z[9] = z[9].float().add(2.0 ** 14).to(dt)
    z[10] = z[10].float().mul(2.0 ** 11).to(dt)
    z[11] = low
    z[12, ::2] = 0.0
    z[12, 1::2] = -0.0
    tokens = torch.tensor([3, vocab - 1, 5, 299, 2, 0, 1, 1, 5, 7, 9, 11, 1, -1],
                          dtype=torch.int32, device="cuda")
    for top in (0, 1, 50):
        for tau in (1.0, 0.5):
            _check(torch, z, tokens, top, tau, _score(torch, z, tokens, top, tau))
    # a token that is masked
    tokens[0] = 299
    _check(torch, z, tokens, 0, 1.0, _score(torch, z, tokens, 0))


def test_score_outputs(torch):
    """Each output by itself is the same as all together."""
    import paper_2202_06009_amd as zo
    z = _logits(torch, 6, 5000, "bfloat16", seed=1, pad=3)
    tokens = _tokens(torch, z, seed=1)
    logp, stats, values, columns = _score(torch, z, tokens, 9)
    one = torch.empty_like(logp)
    zo.zo_token_logprobs(z, tokens, one)
    assert torch.equal(one, logp)
    one = torch.empty_like(stats)
    zo.zo_token_logprobs(z, stats=one)
    assert torch.equal(one, stats)
    v, c = torch.empty_like(values), torch.empty_like(columns)
    zo.zo_token_logprobs(z, values=v, columns=c)
    assert torch.equal(v, values) and torch.equal(c, columns)


@pytest.mark.parametrize("dtype,vocab", [("bfloat16", 8000), ("float32", 20001),
                                         ("bfloat16", 50257)])
def test_score_same_bits_in_any_batch(torch, dtype, vocab):
    """A row's sums do not depend on the other rows or on how many alternatives are wanted:
    the forms for few rows, many rows and many alternatives."""
    z = _logits(torch, 700, vocab, dtype, seed=8, pad=1)
    tokens = _tokens(torch, z, seed=8)
    many = _score(torch, z, tokens, 20)
    for rows, top in ((3, 20), (700, 0), (3, 0), (5, 300), (700, 300)):
        got = _score(torch, z[:rows], tokens[:rows], top)
        assert torch.equal(got[0], many[0][:rows]) and torch.equal(got[1], many[1][:rows])
        if top:
            assert torch.equal(got[2][:, :20], many[2][:rows])
            assert torch.equal(got[3][:, :20], many[3][:rows])


@pytest.mark.parametrize("tau", [2.0 ** -126, 2.0 ** -20, 2.0 ** 20, 2.0 ** 125, 3e38])
def test_score_extreme_tau(torch, tau):
    """Temperatures near binary32's ends: one logit has everything, or all are alike.  A
    distance over tau that passes binary32 is -infinity."""
    z = _logits(torch, 4, 3000, "float32", seed=2)
    z[1, 5] = -torch.inf
    z[2, :2500] = -torch.inf
    tokens = torch.tensor([7, 5, 2600, 9], dtype=torch.int32, device="cuda")
    tau = float(torch.tensor(tau))
    _check(torch, z, tokens, 5, tau, _score(torch, z, tokens, 5, tau))


@pytest.mark.parametrize("dtype", DTYPES)
def test_score_growing_rows(torch, dtype):
    """Each vector far above the ones before it, and the first ones masked: the sums are moved
    on the way."""
    z = _logits(torch, 3, 9001, dtype, seed=5)
    step = torch.arange(9001, device="cuda") // 500
    z[0] += (step * 100).to(z.dtype)
    z[1, :8500] = -torch.inf
    z[2, 4000:] += 3000
    tokens = torch.tensor([9000, 8700, 4100], dtype=torch.int32, device="cuda")
    _check(torch, z, tokens, 30, 1.0, _score(torch, z, tokens, 30))


def _check_grad(torch, z, tokens, tau, dlogp, dentropy, dz, rows=None):
    import i8_ref as ref
    stats = ref.score(z.double(), None, tau)[1]
    want, off = ref.score_grad(z.double(), tokens, tau, stats, dlogp, dentropy)
    half, tiny = ref.HALF[z.dtype], ref.TINY[z.dtype]
    rows = slice(None) if rows is None else rows
    err = (dz.double() - want).abs()[rows]
    lim = (off + half * (want.abs() + off) + tiny)[rows]
    assert bool((err <= lim).all()), float((err - lim).max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_score_grad(torch, vocab, dtype):
    import paper_2202_06009_amd as zo
    for rows, pad, tau in ((1, 0, 1.0), (6, 3, 0.7), (9, 8, 1.5)):
        z = _logits(torch, rows, vocab, dtype, seed=vocab + rows, pad=pad)
        tokens = _tokens(torch, z, seed=rows)
        stats = _score(torch, z, None, 0, tau)[1]
        g = torch.Generator().manual_seed(rows)
        dlogp = torch.randn(rows, generator=g).cuda()
        dentropy = (torch.randn(rows, generator=g) * 0.1).cuda()
        for a, b in ((dlogp, dentropy), (dlogp, None), (None, dentropy)):
            full = torch.full((rows, vocab + pad), 7.0, dtype=z.dtype, device="cuda")
            dz = full[:, :vocab]
            zo.zo_token_logprobs_grad(z, stats, dz, tokens=None if a is None else tokens, dlogp=a,
                                      dentropy=b, tau=tau)
            _check_grad(torch, z, tokens, tau, a, b, dz)
            assert (full[:, vocab:] == 7.0).all()
        inplace = z.clone(memory_format=torch.preserve_format)
        zo.zo_token_logprobs_grad(inplace, stats, inplace, dentropy=dentropy, tau=tau)
        assert torch.equal(inplace, dz)


@pytest.mark.parametrize("dtype", DTYPES)
def test_score_grad_masks(torch, dtype):
    """Masked columns and rows, rows that count for nothing (not read: NaN there stays
    unseen), NaN in rows that count."""
    import paper_2202_06009_amd as zo
    vocab = 3001
    z = _logits(torch, 9, vocab, dtype, seed=6)
    z[0, 40:] = -torch.inf
    z[1, :-1] = -torch.inf
    z[2] = -torch.inf
    z[3, 2:] = torch.finfo(z.dtype).min
    z[5, 5] = torch.nan
    z[6, 5] = torch.inf
    z[7] = torch.nan
    tokens = torch.tensor([3, vocab - 1, 5, 1, -1, 1, 1, 4, 700], dtype=torch.int32, device="cuda")
    dlogp = torch.tensor([1.0, -2, 1, 0.5, 3, 1, 1, 0, -1], device="cuda")
    dentropy = torch.tensor([0.1, 0.2, 0.3, -0.1, 0, 0.1, 0.1, 0, 0], device="cuda")
    stats = _score(torch, z, None, 0)[1]
    dz = torch.full_like(z, 7.0)
    zo.zo_token_logprobs_grad(z, stats, dz, tokens=tokens, dlogp=dlogp, dentropy=dentropy)
    _check_grad(torch, z, tokens, 1.0, dlogp, dentropy, dz, [0, 1, 2, 3, 4, 8])
    assert not dz[0, 40:].any() and not dz[3, 2:].any() and not dz[2].any() and not dz[4].any() and not dz[7].any()
    assert dz[5:7].isnan().all()


def test_score_grad_by_differences(torch):
    """Against differences of the forward pass in binary32: over 2^-6 of the logits' size
    the relative error of a central difference is about 2^-12."""
    import paper_2202_06009_amd as zo
    rows, vocab, tau = 4, 37, 0.8
    z = torch.randn((rows, vocab), device="cuda") * 2
    tokens = torch.tensor([3, 36, 0, 9], dtype=torch.int32, device="cuda")
    a, b = torch.randn(rows, device="cuda"), torch.randn(rows, device="cuda")

    def value(z):
        logp, stats, _, _ = _score(torch, z, tokens, 0, tau)
        return float((a.double() * logp.double() + b.double() * stats[:, 2].double()).sum())

    dz = torch.empty_like(z)
    stats = _score(torch, z, tokens, 0, tau)[1]
    zo.zo_token_logprobs_grad(z, stats, dz, tokens=tokens, dlogp=a, dentropy=b, tau=tau)
    along = torch.randn_like(z)
    got = (value(z + 2.0 ** -6 * along) - value(z - 2.0 ** -6 * along)) * 2.0 ** 5
    want = float((dz.double() * along.double()).sum())
    assert abs(got - want) <= 2.0 ** -8 * float((dz.double() * along.double()).abs().sum())


def test_score_small_probability_keeps_digits(torch):
    """The token's gradient where its probability is nearly 1: dlogp (1 - p), not 0."""
    import paper_2202_06009_amd as zo
    z = torch.zeros((1, 9), device="cuda")
    z[0, 4] = 20.0
    tokens = torch.tensor([4], dtype=torch.int32, device="cuda")
    stats = torch.tensor([[20.0, 8 * 2.0611536181902037e-9, 3.4628e-7]], device="cuda")
    dz = torch.empty_like(z)
    zo.zo_token_logprobs_grad(z, stats, dz, tokens=tokens, dlogp=torch.ones(1, device="cuda"))
    assert abs(float(dz[0, 4]) / (8 * 2.0611536181902037e-9) - 1) < 2.0 ** -20


def test_score_empty_rows_and_offsets(torch):
    import paper_2202_06009_amd as zo
    none = torch.empty((0, 40), device="cuda")
    _score(torch, none, torch.empty(0, dtype=torch.int32, device="cuda"), 3)
    zo.zo_token_logprobs_grad(none, torch.empty((0, 3), device="cuda"), none.clone(),
                              dentropy=torch.empty(0, device="cuda"))
    zo.zo_token_logprobs(none, stats=torch.empty((0, 3), device="cuda"))
    # offsets beyond 2^32 bytes
    z = torch.zeros((45000, 50257), dtype=torch.bfloat16, device="cuda")
    z[-2:] = _logits(torch, 2, 50257, "bfloat16", seed=3)
    tokens = torch.full((45000,), 17, dtype=torch.int32, device="cuda")
    big = _score(torch, z, tokens, 4)
    small = _score(torch, z[-2:].clone(), tokens[-2:].clone(), 4)
    assert all(torch.equal(a[-2:], b) for a, b in zip(big, small))
    ones = torch.ones(45000, device="cuda")
    want = torch.empty_like(z[-2:])
    zo.zo_token_logprobs_grad(z[-2:].clone(), small[1], want, tokens=tokens[-2:].clone(),
                              dlogp=ones[-2:].clone(), dentropy=ones[-2:].clone())
    zo.zo_token_logprobs_grad(z, big[1], z, tokens=tokens, dlogp=ones, dentropy=ones)
    assert torch.equal(z[-2:], want)


def test_score_stream_and_graph(torch):
    import paper_2202_06009_amd as zo
    z = _logits(torch, 33, 5003, "bfloat16", seed=1, pad=5)
    tokens = _tokens(torch, z, seed=1)
    ones = torch.ones(33, device="cuda")

    def step(stream=None):
        got = _score(torch, z, tokens, 7, stream=stream)
        dz = torch.empty((33, 5003), dtype=z.dtype, device="cuda")
        zo.zo_token_logprobs_grad(z, got[1], dz, tokens=tokens, dlogp=ones, dentropy=ones,
                                  stream=stream)
        return (*got, dz)

    eager = step()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):               # the buffers are filled there too
        other = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(4):
        z.copy_(torch.randn((33, 5003), device="cuda") * (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in held]
        assert all(torch.equal(a, b) for a, b in zip(got, step()))
