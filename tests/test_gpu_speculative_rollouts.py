"""The example drafts, verifies and takes the loss in a row: what it emits is the head's own, and its gradient the formula's."""
import importlib.util
import os

import pytest
import torch

import paper_2203_16340_amd as L

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("speculative_rollouts", os.path.join(ROOT, "examples", "speculative_rollouts.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.fixture(scope="module")
def ran(example):
    return example.run(vocab=700, width=96, requests=9, drafts=3, tokens=20, steps=2)


def test_answers_are_whole_and_their_log_probabilities_the_heads(example, ran):
    for s in ran["steps"]:
        assert s["answers"].shape == (9, 20) and (s["answers"] >= 0).all() and (s["answers"] < 700).all() and (s["length"] == 20).all()
        assert 20 / 4 <= s["rounds"] <= 20
        z = example.positions(ran["features"], ran["first"], s["answers"]) @ s["head"].t()
        want = torch.log_softmax(z.double(), 1).gather(1, s["answers"].flatten()[:, None])[:, 0]
        # (two products of 96 terms of size 3 in 32 bits, in another order: 96 * 2^-24 * 30 of a logit each way, and the log-probability's own 4e-6)
        assert (s["logp"].flatten().double() - want).abs().max() < 4e-4


def test_the_gradient_is_the_formulas_and_the_differences(example, ran):
    s = ran["steps"][0]
    x, y = example.positions(ran["features"], ran["first"], s["answers"]).double(), s["answers"].flatten()
    got = ran["value"][y].double()
    adv = (got - got.mean()) / got.std()
    old = s["logp"].flatten().double()

    def loss(head):
        lp = torch.log_softmax(x @ head.t(), 1)
        r = torch.exp(lp.gather(1, y[:, None])[:, 0] - old)
        entropy = -(lp.exp() * lp).sum(1)
        return (-torch.minimum(r * adv, r.clamp(0.8, 1.2) * adv) - 1e-3 * entropy).mean()

    head = s["head"].double().requires_grad_()
    want = torch.autograd.grad(loss(head), head)[0]
    # (a row's gradient is off by 1e-5 of its terms, which are at most its weight's size times a feature's: 1 / 180 * 4, and 180 rows add up)
    assert (s["grad"].double() - want).abs().max() < 2e-5 * want.abs().max() + 1e-6
    gen = torch.Generator("cuda").manual_seed(3)
    for _ in range(3):
        way = torch.randn(head.shape, device="cuda", dtype=torch.float64, generator=gen)
        h = 1e-4
        diff = (loss(head.detach() + h * way) - loss(head.detach() - h * way)) / (2 * h)
        assert abs(diff.item() - (s["grad"].double() * way).sum().item()) < 1e-3 * abs(diff.item()) + 1e-5


def test_what_the_rollouts_call_stands_in_the_package():
    for name in ("matvec4", "pack4", "quantize4", "draw_tokens", "verify_draft"):
        assert callable(getattr(L, name)) and getattr(L, name).__doc__
