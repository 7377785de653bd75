"""Offsets that descend: the values are those of the answers so cut, and the gradient, in which answers that share tokens would meet, is no
number, the same from call to call."""
import pytest
import torch

import paper_2203_16340_amd as L
from gpu_helpers import DEV

pytestmark = pytest.mark.gpu


def _off(*values):
    return torch.tensor(values, dtype=torch.int64, device=DEV)


@pytest.mark.parametrize("off,rewards", [((0, 10, 5, 12, 15, 18, 20), (-10.0, 0.0, -7.0, -3.0, -3.0, -2.0)),     # tokens 5 to 9 twice
                                         ((8, 5, 12), (0.0, -7.0)), ((30, -4, 20), (0.0, -20.0)), ((5, 5, 4), (0.0, 0.0))])
def test_descending_offsets(off, rewards):
    lp = torch.full((20,), -1.0, device=DEV)
    first = L.preference_loss(lp, None, _off(*off), beta=1.0)
    again = L.preference_loss(lp, None, _off(*off), beta=1.0)
    assert first.rewards.tolist() == list(rewards) and torch.equal(first.rewards, again.rewards) and torch.equal(first.loss, again.loss)
    assert torch.isnan(first.grad).all() and torch.isnan(again.grad).all()
    none = L.preference_loss(lp, None, _off(*off), beta=1.0, grad=False)
    assert none.grad is None and torch.equal(none.rewards, first.rewards) and torch.equal(none.loss, first.loss)


def test_one_place_of_many():
    """Every pair of neighbours is looked at, where there are more than the closing workgroup has threads."""
    pairs, each = 1500, 3
    good = torch.arange(2 * pairs + 1, dtype=torch.int64, device=DEV) * each
    lp = -torch.rand(2 * pairs * each, device=DEV)
    want = L.preference_loss(lp, None, good)
    assert torch.isfinite(want.grad).all()
    for at in (2, 1023, 1024, 2 * pairs - 1, 2 * pairs):
        bad = good.clone()
        bad[at] = bad[at - 1] - 1
        assert torch.isnan(L.preference_loss(lp, None, bad).grad).all()


def test_ascending_once_taken_into_the_tokens():
    lp = torch.full((10,), -1.0, device=DEV)
    r = L.preference_loss(lp, None, _off(-3, -9, 4, 22, 11), beta=1.0)      # 0, 0, 4, 10, 10
    assert r.rewards.tolist() == [0.0, -4.0, -6.0, 0.0] and torch.isfinite(r.grad).all() and (r.grad != 0).all()
    r = L.preference_loss(lp, None, _off(2, 2, 2), beta=1.0)
    assert (r.grad == 0).all() and abs(r.loss.item() - 0.6931472) < 1e-6
