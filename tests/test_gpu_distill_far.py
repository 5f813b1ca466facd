"""The distillation loss where logits lie far from each other, under masks and near the
ends of the type, against the 64-bit oracle within limits of each row's own."""
import numpy as np
import pytest

import logit_bounds as lb

pytestmark = pytest.mark.gpu

LOWEST = {"float32": -lb.FLT_MAX, "float16": -65504.0, "bfloat16": -float.fromhex("0x1.fep127")}


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def _check(torch, dtype, z, vals, cols, *, inplace=False, **kw):
    import paper_2202_06009_amd as zo

    def dev(a, dt):
        return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dt).cuda()
    x = torch.from_numpy(z).to(getattr(torch, dtype)).cuda()
    z = x.double().cpu().numpy()
    loss = torch.full((len(z),), 7.0, device="cuda")
    dz = x if inplace else torch.full_like(x, 7.0)
    f32, i32 = torch.float32, torch.int32
    zo.zo_distill_loss(x, dev(vals, f32), dev(cols, i32), loss, dz, tau=kw.get("tau", 1.0),
                       teacher_lse=dev(kw.get("lse"), f32), labels=dev(kw.get("labels"), i32),
                       kd_weight=kw.get("kd", 1.0), ce_weight=kw.get("ce", 0.0),
                       row_weight=dev(kw.get("weight"), f32))
    loss, dz = loss.double().cpu().numpy(), dz.double().cpu().numpy()
    with np.errstate(all="ignore"):
        want, want_dz, lim, lim_dz = lb.distill(z, vals, cols, dtype, **kw)
        off, off_dz = np.abs(loss - want), np.abs(dz - want_dz)
        # past the end of binary32 within the limit
        ends = np.isinf(loss) & (np.sign(loss) * want + lim >= lb.FLT_MAX)
    bad = ~((loss == want) | (off <= lim) | ends)
    assert not bad.any(), (np.flatnonzero(bad), loss[bad], want[bad], lim[bad])
    bad = ~(off_dz <= lim_dz)
    at = np.argwhere(bad)[:4]
    assert not bad.any(), (at, [(dz[i, j], want_dz[i, j], lim_dz[i, j]) for i, j in at])


# rows in registers, and rows that are read twice
VOCABS = [40, 3001, 50257, 70001, 140001]


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0])
def test_rest_far_below(torch, vocab, tau, dtype):
    """A student that holds all outside S far below S, but not excluded: the loss is finite,
    and where the teacher has nothing there either, its rounding is not made a loss."""
    masks = [-100.0, -1e4, max(-1e9, LOWEST[dtype]), LOWEST[dtype]]
    z, vals, cols, lse, _ = lb.far_rest_rows(vocab, tau, masks, False)
    _check(torch, dtype, z, vals, cols, tau=tau, lse=lse)
    _check(torch, dtype, z, vals, cols, tau=tau, lse=lse, kd=0.7, inplace=True)


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("tau", [1.0, 2.0, 1.5])
def test_large_logits(torch, vocab, tau):
    """Rows at values whose products' units in the last place are many exponents."""
    z, vals, cols, lse, _ = lb.far_rest_rows(vocab, tau, [-1e12, -1e30], False)
    _check(torch, "float32", z, vals, cols, tau=tau, lse=lse)
    _check(torch, "bfloat16", z, vals, cols, tau=tau, lse=lse, inplace=True)
    z, vals, cols, lse, labels = lb.large_rows(vocab, tau)
    for tail in (False, True):
        _check(torch, "float32", z, vals, cols, tau=tau, lse=lse if tail else None)
        _check(torch, "float32", z, vals, cols, tau=tau, lse=lse if tail else None, labels=labels,
               ce=0.5, inplace=True)


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0, 1.5])
def test_lowest_labels_and_slots(torch, vocab, tau):
    """Labels and used slots whose logits are the type's lowest value: excluded only where
    the distance from the largest passes binary32."""
    z, vals, cols, lse, labels = lb.far_rest_rows(vocab, tau, [-50.0, LOWEST["float32"]], True)
    _check(torch, "float32", z, vals, cols, tau=tau, lse=lse, labels=labels, ce=0.5)
    z = np.maximum(z, LOWEST["bfloat16"])
    _check(torch, "bfloat16", z, vals, cols, tau=tau, lse=lse, labels=labels, kd=0.0, ce=1.0)
    z[::3, :] = 0.5                                   # slots at the lowest, the rest not
    z[np.arange(len(z)), cols[:, 1]] = LOWEST["float32"]
    for tail in (False, True):
        _check(torch, "float32", z, vals, cols, tau=tau, lse=lse if tail else None, labels=labels,
               ce=0.5)


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("tau", [1.0, 2.0, 1.5])
def test_masks(torch, vocab, tail, tau):
    for dtype in ("float32", "float16", "bfloat16"):
        z, vals, cols, lse, labels, weight = lb.masked_rows(vocab, tau, LOWEST[dtype])
        for ce in (0.0, 0.5):
            _check(torch, dtype, z, vals, cols, tau=tau, lse=lse if tail else None, labels=labels,
                   ce=ce, weight=weight)


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("tau", [1.0, 2.0, 1.5])
def test_ends_of_the_type(torch, vocab, tail, tau):
    """Largest logits near the ends of binary32, in rows that were read into registers
    before that is known, in place and not."""
    z, vals, cols, lse, labels = lb.extreme_rows(vocab, tau)
    for inplace in (False, True):
        for ce in (0.0, 0.5):
            _check(torch, "float32", z, vals, cols, tau=tau, lse=lse if tail else None,
                   labels=labels, ce=ce, inplace=inplace)


@pytest.mark.parametrize("vocab", VOCABS)
def test_tau_below_the_normal_numbers(torch, vocab):
    """log2(e) / tau passes binary32; q and p are those of the largest logits alone."""
    r = np.random.default_rng(vocab)
    z = -r.integers(0, 3, (4, vocab)).astype(np.float64)
    z[1], z[2], z[3] = z[1] + 2.0, 0.0, z[3] - 5.0
    cols = np.stack([r.permutation(vocab)[:5] for _ in range(4)]).astype(np.int32)
    vals = r.integers(-1, 1, (4, 5)).astype(np.float32)
    for tail in (False, True):
        for ce in (0.0, 0.5):
            _check(torch, "float32", z, vals, cols, tau=2.0 ** -133, ce=ce, labels=cols[:, 1].copy(),
                   lse=np.log(3 * np.ones(4, np.float32)) if tail else None)


@pytest.mark.parametrize("vocab", VOCABS)
def test_not_a_number_is_not_hidden(torch, vocab):
    """A NaN in a used slot, with everything else excluded and mass of the teacher there;
    one outside S; the rows beside them keep theirs."""
    import paper_2202_06009_amd as zo
    z = torch.full((4, vocab), -float("inf"), device="cuda")
    cols = torch.tensor([[3, 7]] * 4, dtype=torch.int32, device="cuda")
    z[:, 3], z[:, 7] = 1.0, 2.0
    z[0, 3] = float("nan")
    z[1, 11] = float("nan")
    z[3, 20] = 0.5
    loss, dz = torch.zeros(4, device="cuda"), torch.zeros_like(z)
    zo.zo_distill_loss(z, torch.ones((4, 2), device="cuda"), cols, loss, dz,
                       teacher_lse=torch.full((4,), 2.0, device="cuda"))
    assert torch.isnan(loss).tolist() == [True, True, False, False]
    assert loss[2] == float("inf") and torch.isfinite(loss[3])
    assert torch.isfinite(dz[2:]).all()
