"""More rows of logits than one launch holds: rows that repeat have the results of the
first of them, bit for bit."""
import pytest

pytestmark = pytest.mark.gpu

ROWS = (1 << 24) + 777         # of 256 threads each: 2^32 and more


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _repeated(t, rows):
    return t.repeat((rows + len(t) - 1) // len(t), *([1] * (t.dim() - 1)))[:rows].contiguous()


def _all_equal(torch, got, first):
    """Every row of got is the row of `first` that it repeats."""
    n, whole = len(first), len(got) // len(first) * len(first)
    view = got[:whole].view(-1, *first.shape)
    return bool((view == first).all()) and torch.equal(got[whole:], first[:len(got) - whole])


def test_top_logits(torch):
    import paper_2202_06009_amd as zo
    n, vocab, top = 1009, 5, 2
    first = torch.randn((n, vocab), device="cuda").bfloat16()

    def run(z):
        values = torch.full((len(z), top), 7.0, device="cuda")
        columns = torch.full((len(z), top), -7, dtype=torch.int32, device="cuda")
        lse = torch.full((len(z),), 7.0, device="cuda")
        zo.zo_top_logits(z, values, columns, lse)
        return values, columns, lse
    want = run(first)
    assert torch.equal(want[0], torch.topk(first.float(), top, dim=1).values)
    for got, one in zip(run(_repeated(first, ROWS)), want):
        assert _all_equal(torch, got, one)


def test_distill(torch):
    import paper_2202_06009_amd as zo
    n, vocab, top = 1009, 5, 2
    z = torch.randn((n, vocab), device="cuda").half()
    values = torch.randn((n, top), device="cuda")
    columns = torch.randint(0, vocab, (n, top), dtype=torch.int32, device="cuda")
    lse = values.logsumexp(1) + 0.3
    labels = torch.randint(0, vocab, (n,), dtype=torch.int32, device="cuda")
    weight = torch.randn(n, device="cuda")
    ins = (z, values, columns, lse, labels, weight)

    def run(z, values, columns, lse, labels, weight):
        loss, dz = torch.full((len(z),), 7.0, device="cuda"), torch.full_like(z, 7.0)
        zo.zo_distill_loss(z, values, columns, loss, dz, teacher_lse=lse, labels=labels,
                           row_weight=weight, ce_weight=0.5)
        return loss, dz
    want = run(*ins)
    assert torch.isfinite(want[0]).all() and torch.isfinite(want[1]).all()
    for got, one in zip(run(*(_repeated(t, ROWS) for t in ins)), want):
        assert _all_equal(torch, got, one)
