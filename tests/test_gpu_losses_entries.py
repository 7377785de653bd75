"""Every entry of the gradients against 64 bits, each to its own size: a zero, or what stood there before, in place of a small probability
shows.  The row lengths are those at which another kernel takes over; every gradient goes into memory that holds NaN.

Bounds: a probability is known to 2e-5 of itself (an argument of at most ~40 with two roundings, ~100 dependent additions), the policy's slope
to 2e-5 of its size by the log-probability in it, the entropy's log p_j + H to 2e-5 of |log p_j| + H + 1, the teacher's shares to 2e-5, their rest's
to 2e-5 of 1.  A gradient is rounded once to its type."""
import numpy as np
import pytest
import torch

import paper_2203_16340_amd as L
from gpu_helpers import DEV
from test_gpu_losses import HALF_UNIT, SMALLEST
from test_gpu_losses_shapes import CHUNKS

pytestmark = pytest.mark.gpu

WEIGHT = 64.0            # lifts gradients of f16 out of its subnormal numbers


def near(got, want, size):
    """size: of the terms that an entry is the sum of"""
    off = (got.double() - want).abs() - (1.01 * HALF_UNIT[got.dtype] * want.abs() + 6e-5 * size + SMALLEST[got.dtype])
    assert not got.isnan().any() and not (off > 0).any(), (off.max().item(), (off > 0).sum().item())


def rows_of(rows, vocab, dtype, shift, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    room = torch.empty(rows, vocab + 2 * shift, dtype=dtype, device=DEV)
    z = room[:, shift:shift + vocab]
    z.copy_((3 * torch.randn(rows, vocab, device=DEV, generator=g)).to(dtype))
    y = torch.randint(0, vocab, (rows,), device=DEV, generator=g)
    y[:3] = torch.tensor([0, vocab - 1, vocab // 2], device=DEV)
    return z, y, g


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows", [3, 64, 66])
@pytest.mark.parametrize("chunks", CHUNKS)
def test_every_entry(chunks, rows, dtype):
    per = 16 // torch.tensor([], dtype=dtype).element_size()
    shift = 0 if rows == 64 else 3
    vocab = chunks * per + shift
    z, y, g = rows_of(rows, vocab, dtype, shift, chunks + rows)
    at = torch.arange(rows, device=DEV)
    lp = torch.log_softmax(z.double() / 0.9, 1)
    p, s = lp.exp(), 1 / 0.9
    H = -(p * lp).sum(1)
    logp = lp[at, y]

    def out():
        return torch.full_like(z, torch.nan)

    def expected(slope, c, W):
        """W (slope (1[j = y] - p) + c p (log p + H)), and the size of its terms"""
        want = -slope[:, None] * p
        size = slope.abs()[:, None] * p
        want[at, y] += slope
        size[at, y] += slope.abs()
        if c is not None:
            want = want + c[:, None] * p * (lp + H[:, None])
            size = size + c.abs()[:, None] * p * (lp.abs() + H[:, None] + 1)
        return W * s * want, W * s * size

    d = WEIGHT * (0.5 + torch.rand(rows, device=DEV, generator=g))
    e = WEIGHT * (torch.rand(rows, device=DEV, generator=g) - 0.5)
    t = L.token_logprob(z, y, temperature=0.9, entropy=True)
    near(L.token_logprob_grad(z, y, t, d, temperature=0.9, grad=out()), *expected(d.double(), None, 1.0))
    near(L.token_logprob_grad(z, y, t, d, d_entropy=e, temperature=0.9, grad=out()), *expected(d.double(), -e.double(), 1.0))

    adv = 0.5 + torch.rand(rows, device=DEV, generator=g)
    old = (logp - 0.1 * torch.rand(rows, device=DEV, generator=g)).float()
    w = torch.full((rows,), WEIGHT, device=DEV)
    slope = -torch.exp(logp - old.double()) * adv.double()
    for coef in (0.0, 0.3):
        r = L.policy_loss(z, y, old, adv, weight=w, entropy_coef=coef, temperature=0.9, grad=out())
        near(r.grad, *expected(slope, torch.full_like(slope, coef) if coef else None, WEIGHT))

    top = min(vocab, 40)
    index = torch.as_tensor(np.stack([np.random.default_rng(chunks + r).choice(vocab, top, replace=False) for r in range(rows)])).to(DEV)
    a = torch.randn(rows, top, device=DEV, generator=g) + 3
    for lse in (None, torch.logsumexp(a / 0.9, 1) + 0.2):
        r = L.distill_loss(z, index, a, teacher_lse=lse, weight=w, temperature=0.9, grad=out())
        scaled = a.double() / 0.9
        q = torch.exp(scaled - (torch.logsumexp(scaled, 1) if lse is None else lse.double())[:, None])
        full = torch.zeros_like(p).scatter_(1, index, q)
        inside = torch.zeros_like(p, dtype=torch.bool).scatter_(1, index, True)
        want, size = p - full, p + full
        if lse is not None and vocab > top:
            rest, t = 1 - q.sum(1, keepdim=True), p.masked_fill(inside, 0).sum(1, keepdim=True)
            want = torch.where(inside, want, p * (1 - rest / t))
            size = torch.where(inside, size, p * (1 + (1 + rest) / t))
        near(r.grad, WEIGHT * s * want, WEIGHT * s * size)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [3, 2003, 33003, 70001])
def test_rows_that_do_not_count_are_cleared(vocab, dtype):
    for rows in (5, 70):
        z, y, g = rows_of(rows, vocab, dtype, 3, vocab)
        y[1] = -1
        one = torch.ones(rows, device=DEV)
        w = one.clone()
        w[3] = 0
        index, a = torch.randint(0, vocab, (rows, 3), device=DEV, generator=g), torch.randn(rows, 3, device=DEV, generator=g)
        t = L.token_logprob(z, y)
        room = [torch.full_like(z, torch.nan) for _ in range(3)]
        L.token_logprob_grad(z, y, t, w, grad=room[0])
        L.policy_loss(z, y, -one, one, weight=w, clip_low=1.0, clip_high=1e9, grad=room[1])
        L.distill_loss(z, index, a, weight=w, grad=room[2])
        for k, r in enumerate(room):
            assert torch.isfinite(r).all() and (r[3] == 0).all() and (k == 2 or (r[1] == 0).all()) and (r[0] != 0).any()
