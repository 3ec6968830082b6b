"""The preference loss's oracle where h is infinite: a target whose logit is -infinity."""
import numpy as np
import pytest

from oracle.prefer import prefer_loss


@pytest.mark.parametrize("smoothing,row,loss", [(0.0, 1, 0.0), (0.0, 0, np.inf), (1.0, 0, 0.0), (1.0, 1, np.inf), (0.25, 1, np.inf)])
def test_a_term_without_weight_is_left_out(smoothing, row, loss):
    x = np.zeros((2, 4))
    x[row, 2] = -np.inf
    with np.errstate(divide="ignore"):
        r = prefer_loss([1, 1], x, [2, 2], ref_logp=np.zeros(2), smoothing=smoothing)
    assert r.loss == loss and np.isfinite(r.grad).all()
