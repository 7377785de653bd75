"""Temperatures at the ends of what is taken: the formulas hold there, with masks, and what 32 bits cannot hold is refused."""
import numpy as np
import pytest
import torch

import losses_reference as ref
import paper_2203_16340_amd as L
from gpu_helpers import DEV
from test_gpu_losses import dev, host, logits_of, near_values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("temperature", [1e-30, 1e-6, 1e6, 1e30, 1e38, 1e39, 1e45, 1e46, 1e300])
@pytest.mark.parametrize("vocab", [9, 1030, 70001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_rows(vocab, dtype, temperature):
    z = logits_of(4, vocab, dtype, seed=21)
    z[0, 2:] = -torch.inf
    z[1, ::2] = -torch.inf
    z[2, 1:] = -3.0
    z[2, 0] = 5.0
    y = np.array([0, 1, 0, vocab - 1])
    s = 1 / temperature
    zd, yd = z.to(DEV), dev(y, torch.int64)
    t = L.token_logprob(zd, yd, temperature=temperature, entropy=True)
    p = L.policy_loss(zd, yd, torch.zeros(4, device=DEV), torch.zeros(4, device=DEV), temperature=temperature, entropy=True)
    want = ref.token_logprob(host(z), y, s)
    for logp, H in ((t.logp, t.entropy), (p.logp, p.entropy)):
        near_values(logp, want[0].astype(np.float32))
        near_values(H, want[2])
    g = L.token_logprob_grad(zd, yd, t, torch.ones(4, device=DEV), temperature=temperature)
    assert torch.isfinite(g).all()
    r = ref.token_grad(host(z), y, s, np.ones(4))
    assert np.allclose(host(g), r, rtol=0.01, atol=1e-5 * s + 1e-37)


def test_refused():
    z, y = torch.zeros(2, 5, device=DEV), torch.zeros(2, dtype=torch.int64, device=DEV)
    f = torch.zeros(2, device=DEV)
    t = L.token_logprob(z, y)
    for temperature in (1e-39, 4e-39, 1e-300):
        for call in (lambda: L.token_logprob(z, y, temperature=temperature), lambda: L.token_logprob_grad(z, y, t, f, temperature=temperature),
                     lambda: L.policy_loss(z, y, f, f, temperature=temperature),
                     lambda: L.distill_loss(z, y[:, None], f[:, None], temperature=temperature)):
            with pytest.raises(L.LbfgsbError, match="temperature"):
                call()
