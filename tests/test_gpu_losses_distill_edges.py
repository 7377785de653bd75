"""Distillation to students whose rows, or entries, are held at the type's lowest or largest value or at -1e9."""
import numpy as np
import pytest
import torch

import losses_reference as ref
import paper_2203_16340_amd as L
from gpu_helpers import DEV
from test_gpu_losses import TYPES, dev, host, logits_of, near_grad, near_values

pytestmark = pytest.mark.gpu


def teacher(rows, vocab, top, seed=0):
    rng = np.random.default_rng(seed)
    index = np.stack([rng.choice(vocab, top, replace=False) for _ in range(rows)])
    a = dev(rng.normal(size=(rows, top)) * 2 + 4)
    return index, a


def off_the_entries(z, index, a, lse, s):
    """Gradient of a row off the entries, the rest's outcome counted: s (p_j - r w_j / sum w), w from differences to the rest's largest
    logit (at the type's lowest value its log-sum-exp, in any number of bits here, says nothing about its entries)."""
    inside = np.zeros(len(z), dtype=bool)
    inside[index] = True
    rest = max(0.0, 1.0 - np.exp(a * s - lse).sum())
    u = z[~inside] * s
    w = np.exp(u - u.max())
    return inside, s * (np.exp(ref.softmax_row(z, s)[1][~inside]) - rest * w / w.sum())


@pytest.mark.parametrize("temperature", [1.0, 0.7, 1.5])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab,top", [(5, 9, 3), (5, 1030, 64), (70, 1030, 5), (5, 70001, 30), (66, 70001, 30)])
def test_students_held_at_one_value(rows, vocab, top, rest, dtype, temperature):
    z = logits_of(rows, vocab, dtype, seed=3)
    z[0] = torch.finfo(dtype).min                    # a uniform student
    z[1] = torch.finfo(dtype).max
    z[2] = -1e9 if dtype != torch.float16 else -3e4
    index, a = teacher(rows, vocab, top)
    z[3, index[3]] = torch.finfo(dtype).min          # the entries alone
    z[4] = torch.finfo(dtype).min                    # all but the entries
    z[4, index[4]] = torch.linspace(-2, 2, top).to(dtype)
    s = 1 / temperature
    lse = dev(np.logaddexp.reduce(host(a) * s, axis=1) + 0.3) if rest else None
    r = L.distill_loss(z.to(DEV), torch.as_tensor(index).to(DEV), a, teacher_lse=lse, temperature=temperature)
    few = 5
    total, loss, grad = ref.distill(host(z)[:few], index[:few], host(a)[:few], None if lse is None else host(lse)[:few], np.ones(few), s, 1.0)
    if rest:
        for k in range(few):
            inside, off = off_the_entries(host(z)[k], index[k], host(a)[k], host(lse)[k], s)
            grad[k, ~inside] = off
    # (log q and log p are off by 1e-5 each, and q and the rest by as much of itself, under logarithms of at most ~20 in rows 0 to 2; in
    # the others of as much as the type holds, where the loss may pass 32 bits)
    near_values(r.row_loss[:3], loss[:3], 12)
    with np.errstate(over="ignore"):
        want = loss[3:].astype(np.float32)
    assert np.allclose(host(r.row_loss[3:few]), want, rtol=2e-5, atol=2.4e-4)
    near_grad(r.grad[:few], grad, s)
    assert torch.isfinite(r.row_loss[[0, 1, 2]]).all()
