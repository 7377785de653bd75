"""A gradient written over logits that another operation keeps for its own way back is noticed, as one of torch's operations in place is."""
import pytest
import torch

import paper_2203_16340_amd as L
from gpu_helpers import DEV

pytestmark = pytest.mark.gpu

ROWS, VOCAB = 4, 33


def _calls():
    y = torch.tensor([0, 5, 32, -1], device=DEV)
    one = torch.ones(ROWS, device=DEV)
    index, a = torch.arange(3, device=DEV).repeat(ROWS, 1), torch.zeros(ROWS, 3, device=DEV)
    return {"token": lambda z, g: L.token_logprob_grad(z, y, L.token_logprob(z, y), one, grad=g),
            "policy": lambda z, g: L.policy_loss(z, y, -one, one, grad=g).grad,
            "distill": lambda z, g: L.distill_loss(z, index, a, grad=g).grad}


@pytest.mark.parametrize("name", ["token", "policy", "distill"])
def test_in_place_on_logits_that_were_kept(name):
    call = _calls()[name]
    x = torch.randn(ROWS, VOCAB, device=DEV, requires_grad=True)
    logits = torch.tanh(x)                               # (keeps its result)
    z = logits.detach()
    before = z._version
    g = call(z, z)
    assert z._version > before
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        logits.backward(g)
    # where nobody keeps them the gradient goes on as ever
    w = torch.randn(VOCAB, 7, device=DEV, requires_grad=True)
    h = torch.randn(ROWS, 7, device=DEV)
    logits = h @ w.t()
    z = logits.detach()
    want = call(z, True)
    logits.backward(call(z, z))
    assert torch.equal(z, want) and torch.allclose(w.grad, want.t() @ h, rtol=1e-4, atol=1e-5)


@pytest.mark.parametrize("name", ["token", "policy", "distill"])
def test_the_logits_are_only_read_otherwise(name):
    call = _calls()[name]
    z = torch.randn(ROWS, VOCAB, device=DEV)
    out = torch.empty_like(z)
    before, there = z._version, out._version
    call(z, True)
    call(z, out)
    assert z._version == before and out._version > there


def test_tensors_of_inference_mode():
    with torch.inference_mode():
        z = torch.randn(ROWS, VOCAB, device=DEV)
    for call in _calls().values():
        mine = z.clone()
        want = call(z, True)
        assert torch.equal(call(mine, mine), want)
    with torch.inference_mode():
        for call in _calls().values():
            mine = z.clone()
            call(mine, mine)
