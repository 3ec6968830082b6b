"""The preference loss at the ends of its range: targets of logits that are -infinity, gradients that are
part of wider rows."""
import numpy as np
import pytest

from oracle.prefer import prefer_loss

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("smoothing", [0.0, 0.25, 1.0])
@pytest.mark.parametrize("row", [1, 4])      # of the chosen answer of pair 0, of the rejected one of pair 1
def test_targets_without_weight(gpu, row, smoothing):
    """A target's logit of -infinity makes h infinite; a term whose weight is zero is not in the loss, other
    pairs' losses and all gradients are finite.  Rows of 64 logits of at most 4: a log probability is off by
    2^-18 at most, a loss of one of three pairs by 2 rows of that, an element by its own 2^-18 and 2^-23."""
    import torch
    import paper_2609_31224_amd as a2t
    rng, rows = np.random.default_rng(row), [2, 1, 1, 1, 2, 2]
    pol = np.clip(rng.standard_normal((9, 64)), -4, 4).astype(np.float32)
    t = rng.integers(0, 64, 9).astype(np.int32)
    pol[row, t[row]] = -np.inf
    lp = rng.uniform(-5, -3, 9).astype(np.float32)
    with np.errstate(divide="ignore"):
        want = prefer_loss(rows, pol, t, ref_logp=lp, beta=0.5, smoothing=smoothing)
    h = a2t.a2t_prefer_create(9, 64, a2t.A2T_F32)
    try:
        losses, x = torch.full((3,), 7.0, device="cuda"), torch.from_numpy(pol).to("cuda")
        ratios, grad = torch.full((6,), 7.0, device="cuda"), torch.full_like(x, 7.0)
        a2t.a2t_prefer_loss(h, rows, x, torch.from_numpy(t).to("cuda"), losses, ref_logp=torch.from_numpy(lp).to("cuda"), beta=0.5, smoothing=smoothing,
                            ratios=ratios, grad=grad)
        torch.cuda.synchronize()
        got, r = losses.cpu().double().numpy(), ratios.cpu().double().numpy()
        gone = np.isinf(want.ratios)
        assert gone.sum() == 1 and np.array_equal(np.isneginf(r), np.isneginf(want.ratios))
        assert (np.abs(r - want.ratios)[~gone] <= 2 * 2.0 ** -18 + 2.0 ** -23 * 20).all()
        assert got[1] == want.margin and abs(got[2] - want.won) <= 2.0 ** -24
        if np.isinf(want.loss):
            assert got[0] == np.inf
        else:
            assert abs(got[0] - want.loss) <= 2.0 ** -17 + 2.0 ** -23 * want.loss
        assert (np.abs(grad.cpu().double().numpy() - want.grad) <= 2.0 ** -18).all()
    finally:
        a2t.a2t_prefer_destroy(h)


def test_a_part_of_wider_rows_takes_no_gradient(gpu):
    """Columns beside the gradient's tensor would be zeroed: such a view is refused and nothing is written, while the
    rows with all their columns, a tensor of the vocabulary's columns, and views as inputs are taken."""
    import torch
    import paper_2609_31224_amd as a2t
    vocab, rows = 60, [3, 2]
    h = a2t.a2t_prefer_create(5, vocab, a2t.A2T_F32)
    wide = torch.full((5, 128), 7.0, device="cuda")
    target, lp = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.full((5,), -4.0, device="cuda")
    losses = torch.full((3,), 7.0, device="cuda")
    view = wide[:, :vocab]
    try:
        for policy, grad in ((torch.zeros((5, 128), device="cuda"), view), (view, view), (torch.zeros((5, 128), device="cuda"), wide[:, :119]),
                             (torch.zeros((1, 128), device="cuda"), wide[:1, :vocab])):
            with pytest.raises(ValueError, match="zeroed"):
                a2t.a2t_prefer_loss(h, rows if len(policy) == 5 else [1, 0], policy, target[:len(policy)], losses, ref_logp=lp[:len(policy)], grad=grad)
        torch.cuda.synchronize()
        assert (wide == 7).all() and (losses == 7).all()
        a2t.a2t_prefer_loss(h, rows, view, target, losses, ref_logp=lp)
        a2t.a2t_prefer_loss(h, rows, view, target, losses, ref_logp=lp, grad=torch.empty((5, 128), device="cuda"))
        torch.cuda.synchronize()
        assert (wide == 7).all() and torch.isfinite(losses).all()
        close = torch.full((5, 64), 7.0, device="cuda")
        a2t.a2t_prefer_loss(h, rows, close, target, losses, ref_logp=lp, grad=close[:, :vocab])
        a2t.a2t_prefer_loss(h, rows, wide, target, losses, ref_logp=lp, grad=wide)
        torch.cuda.synchronize()
        assert not wide[:, vocab:].any() and not close[:, vocab:].any() and torch.equal(wide[:, :vocab], close[:, :vocab])
    finally:
        a2t.a2t_prefer_destroy(h)
