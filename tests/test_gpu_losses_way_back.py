"""The way back of token log-probabilities at temperatures that are no power of two, on rows where that shows: held whole at the type's lowest or
largest value, at -1e9, or far from 0.  There (z - m) s keeps its digits and z s - lse does not.

Bounds, from the arithmetic: an entry's exponent (z_j - m) s has an argument of at most ~40 where it counts and two roundings, S at most ~100
dependent additions, so p_j is known to 2e-5 of itself; with the entropy's term p_j (log p_j + H) each of log p_j and H to 2e-5 of its size and of 1."""
import numpy as np
import pytest
import torch

import losses_reference as ref
import paper_2203_16340_amd as L
from gpu_helpers import DEV
from test_gpu_losses import EPS, HALF_UNIT, SMALLEST, TYPES, dev, host, logits_of, near_values

pytestmark = pytest.mark.gpu

TEMPERATURES = [0.6, 0.7, 1.1, 1.2, 1.5, 2.0, 3.0]


def rows_of(dtype, vocab):
    low, most = torch.finfo(dtype).min, torch.finfo(dtype).max
    z = logits_of(9, vocab, dtype, seed=11)
    z[0, :] = low
    z[1, :] = most
    z[2, :] = -1e9 if dtype != torch.float16 else -3e4
    z[3] = (z[3].float() + 1e4).to(dtype)
    z[4] = (z[4].float() - 1e4).to(dtype)
    z[5, 1:] = low
    z[6, ::2] = low
    z[7, :] = -torch.inf
    y = np.array([0, vocab - 1, vocab // 2, 1, vocab - 1, 0, 1, 0, vocab // 3])
    return z, y


def check(got, z, y, s, d, e, rows=slice(None)):
    want = ref.token_grad(host(z), y, s, d, e)
    got = host(got)
    room = np.zeros(z.shape)
    for r in range(len(y)):
        lse, lp, H = ref.softmax_row(host(z)[r], s)
        if lse == -np.inf:
            continue
        p = np.exp(lp)
        size = abs(d[r])
        if e is not None:
            size = size + abs(e[r]) * (np.where(p > 0, np.abs(lp), 0.0) + H + 1)
        room[r] = 2e-5 * s * p * size
        room[r, y[r]] += 4 * EPS * s * abs(d[r])
    bound = room + (1.01 * HALF_UNIT[z.dtype] + 1e-5) * np.abs(want) + SMALLEST[z.dtype]
    off = (np.abs(got - want) - bound)[rows]
    assert np.isfinite(got[rows]).all() and off.max() <= 0, (off.max(1), np.abs(want[rows]).max(1))


@pytest.mark.parametrize("temperature", TEMPERATURES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [9, 1030, 70001])
def test_rows_at_the_ends_of_the_type(vocab, dtype, temperature):
    z, y = rows_of(dtype, vocab)
    s = 1 / temperature
    rng = np.random.default_rng(3)
    d32, e32 = dev(32 * (1 + rng.random(9))), dev(16 * (1 + rng.random(9)))
    zd, yd = z.to(DEV), dev(y, torch.int64)
    t = L.token_logprob(zd, yd, temperature=temperature, entropy=True)
    want = ref.token_logprob(host(z), y, s)
    near_values(t.logp, want[0])
    near_values(t.entropy, want[2])
    check(L.token_logprob_grad(zd, yd, t, d32, temperature=temperature), z, y, s, host(d32), None)
    check(L.token_logprob_grad(zd, yd, t, d32, d_entropy=e32, temperature=temperature), z, y, s, host(d32), host(e32))


@pytest.mark.parametrize("temperature", TEMPERATURES)
@pytest.mark.parametrize("dtype", TYPES)
def test_from_the_log_sum_exp_alone(dtype, temperature):
    """Without the maxima and sums a gradient is right, or where lse and lse_rest do not tell it is no number."""
    vocab = 1030
    z, y = rows_of(dtype, vocab)
    s = 1 / temperature
    zd, yd = z.to(DEV), dev(y, torch.int64)
    t = L.token_logprob(zd, yd, temperature=temperature)
    d = np.full(9, 32.0)
    plain = L.TokenLogprob(*t)
    assert plain.stats is None
    got = L.token_logprob_grad(zd, yd, plain, dev(d), temperature=temperature)
    wide = dtype != torch.float16                    # (its lowest value leaves lse all its digits)
    lost = [0, 1] if wide and temperature != 2.0 else []
    assert torch.isnan(got[lost].float()).all()
    check(got, z, y, s, d, None, [r for r in range(9) if r not in lost])
