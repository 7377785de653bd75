"""Rows without entries of the teacher give zeros, whatever the teacher's log-sum-exp and the student's logits are."""
import numpy as np
import pytest
import torch

import losses_reference as ref
import paper_2203_16340_amd as L
from gpu_helpers import DEV
from test_gpu_losses import host, logits_of, near_grad, near_values
from test_gpu_losses_distill_edges import teacher

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lse", [-np.inf, np.nan, -100.0, np.inf, 1.0])
@pytest.mark.parametrize("rows,vocab", [(3, 9), (3, 1030), (70, 1030), (3, 70001), (66, 70001)])
def test_rows_without_entries(rows, vocab, lse):
    z = logits_of(rows, vocab, torch.float32, seed=4)
    index, a = teacher(rows, vocab, 4)
    index[0] = -1
    a[1] = -torch.inf
    z[1, 3] = torch.nan                              # (whatever the row holds)
    index[1, 2] = -7
    given = torch.logsumexp(a, 1) + 0.3
    given[:2] = lse
    w = torch.full((rows,), 0.5, device=DEV)
    for teacher_lse in (given, None):
        room = torch.full((rows, vocab), 7.0, device=DEV)
        r = L.distill_loss(z.to(DEV), torch.as_tensor(index).to(DEV), a, teacher_lse=teacher_lse, weight=w, grad=room)
        assert (r.row_loss[:2] == 0).all() and (r.grad[:2] == 0).all()
        assert torch.isfinite(r.loss) and torch.isfinite(r.grad).all() and (r.grad[2].abs() > 0).any()
        none = L.distill_loss(z.to(DEV), torch.as_tensor(index).to(DEV), a, teacher_lse=teacher_lse, weight=w, grad=False)
        assert (none.row_loss[:2] == 0).all() and torch.isfinite(none.loss)
        # the other rows are what they are
        total, loss, grad = ref.distill(host(z)[2:3], index[2:3], host(a)[2:3], None if teacher_lse is None else host(given)[2:3], np.full(1, 0.5), 1.0, 1.0)
        near_values(r.row_loss[2:3], loss, 12)
        near_grad(r.grad[2:3], grad, 0.5)
