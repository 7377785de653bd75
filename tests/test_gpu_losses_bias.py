"""Errors of log-probabilities that have one sign: they add up over an answer's tokens, where rounding averages out.

The exponent is (z - m) s log2(e).  With its factor rounded to 32 bits, relative error f (1.3e-8 at temperature 1, up to 6e-8 at others), ln S
is off by f E_p|log(p/p_max)| in every row, here 5 to 10 times f.  What a thread's own largest entry leaves of that is a quarter or less;
the rest has either sign: the roundings of some hundred terms that count, and of the result (2.4e-7 at most for |logp| < 8, the mean of 2048
rows 2e-9), and the instruction's own mean error, less than 1e-8 of a term.  3e-8, half of one rounding to 32 bits, is asked for."""
import math

import pytest
import torch

import paper_2203_16340_amd as L
from gpu_helpers import DEV

pytestmark = pytest.mark.gpu

ROWS = 2048


@pytest.mark.parametrize("temperature", [1.0, 0.7, 0.8, 1.3, 1.7])
@pytest.mark.parametrize("dtype,vocab", [(torch.bfloat16, 65536), (torch.float32, 32768), (torch.float16, 2000)])
def test_log_probabilities_have_no_bias(dtype, vocab, temperature):
    g = torch.Generator(device=DEV).manual_seed(vocab)
    z = (2.2 * torch.randn(ROWS, vocab, device=DEV, generator=g)).to(dtype)
    y = torch.randint(0, vocab, (ROWS,), device=DEV, generator=g)
    z[torch.arange(ROWS, device=DEV), y] = (math.log(vocab) + 1.5 + 1.5 * torch.randn(ROWS, device=DEV, generator=g)).to(dtype)
    want, entropy = [], []
    for at in range(0, ROWS, 256):
        lp = torch.log_softmax(z[at:at + 256].double() / temperature, 1)
        want.append(lp.gather(1, y[at:at + 256, None])[:, 0])
        entropy.append(-(lp.exp() * lp).sum(1))
    want, entropy = torch.cat(want), torch.cat(entropy)
    t = L.token_logprob(z, y, temperature=temperature, entropy=True)
    few = torch.cat([L.token_logprob(z[at:at + 64], y[at:at + 64], temperature=temperature).logp for at in range(0, ROWS, 64)])
    p = L.policy_loss(z, y, torch.zeros_like(t.logp), torch.zeros_like(t.logp), temperature=temperature)
    for logp in (t.logp, few, p.logp):
        assert abs((logp.double() - want).mean().item()) <= 3e-8
    assert abs((t.entropy.double() - entropy).mean().item()) <= 3e-7       # (up to 10 of such terms, and their sum)
