"""Masks at the type's lowest value, at temperatures so low that a difference to them, times the part of the exponents' factor that 32 bits
leave over, is past the end of 32 bits: such entries weigh nothing, whether that part is below 0 (3e-8, 1e-12, 1e-30) or above (3e-9, 5e-39)."""
import numpy as np
import pytest
import torch

import losses_reference as ref
import paper_2203_16340_amd as L
from gpu_helpers import DEV
from test_gpu_losses import TYPES, dev, host, logits_of, near_values

pytestmark = pytest.mark.gpu

TEMPERATURES = [3e-8, 1e-12, 1e-30, 3e-9, 5e-39]


def held_low(rows, vocab, dtype):
    """(logits, labels): the label is the only entry, the last one, one of the others' ties, one of all"""
    low = torch.finfo(dtype).min
    z = logits_of(rows, vocab, dtype, seed=31)
    z[0, 1:] = low
    z[1, :-1] = low
    z[2, ::2] = low
    z[2, 1::2] = 1.0
    z[3, :] = low
    z[4, vocab // 2:] = low
    z[4, 2] = 50.0
    y = np.zeros(rows, dtype=np.int64)
    y[:5] = 0, vocab - 1, 1, vocab // 2, 2
    y[5:] = z[5:].float().argmax(1).numpy()
    return z, y


@pytest.mark.parametrize("temperature", TEMPERATURES)
@pytest.mark.parametrize("rows,vocab", [(5, 9), (5, 1030), (5, 70001), (70, 1030), (70, 70001)])
@pytest.mark.parametrize("dtype", TYPES)
def test_log_probabilities_and_policy(dtype, rows, vocab, temperature):
    z, y = held_low(rows, vocab, dtype)
    s = 1 / temperature
    zd, yd, zeros = z.to(DEV), dev(y, torch.int64), torch.zeros(rows, device=DEV)
    want = ref.token_logprob(host(z), y, s)
    t = L.token_logprob(zd, yd, temperature=temperature, entropy=True)
    plain = L.token_logprob(zd, yd, temperature=temperature)
    p = L.policy_loss(zd, yd, zeros, zeros, temperature=temperature, entropy=True)
    for logp in (t.logp, plain.logp, p.logp):
        near_values(logp, want[0])
    for entropy in (t.entropy, p.entropy):
        near_values(entropy, want[2])
    if dtype != torch.float16:                            # (whose gradients, of the size 1 / temperature, have no room there)
        g = L.token_logprob_grad(zd, yd, t, torch.ones(rows, device=DEV), temperature=temperature)
        assert np.allclose(host(g), ref.token_grad(host(z), y, s, np.ones(rows)), rtol=0.01, atol=1e-5 * s)


@pytest.mark.parametrize("temperature", TEMPERATURES)
@pytest.mark.parametrize("rows,vocab", [(5, 30), (5, 70001), (70, 1030)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rest", [False, True])
def test_distillation(rest, dtype, rows, vocab, temperature):
    """The teacher's first entry has all its weight, and so has the student's there: no loss."""
    top = 7
    z = torch.full((rows, vocab), torch.finfo(dtype).min, dtype=dtype)
    rng = np.random.default_rng(rows + vocab)
    index = np.stack([rng.choice(vocab, top, replace=False) for _ in range(rows)])
    z[torch.arange(rows), torch.as_tensor(index[:, 0])] = 2.0
    a = np.concatenate([np.zeros((rows, 1)), -1 - rng.random((rows, top - 1))], 1)
    lse = torch.zeros(rows, device=DEV) if rest else None
    r = L.distill_loss(z.to(DEV), torch.as_tensor(index).to(DEV), dev(a), teacher_lse=lse, temperature=temperature, grad=dtype != torch.float16)
    assert torch.equal(r.row_loss, torch.zeros(rows, device=DEV)) and r.loss == 0
    if r.grad is not None:
        assert (r.grad == 0).all()
