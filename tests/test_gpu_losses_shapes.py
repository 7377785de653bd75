"""The losses on logits at the row lengths where another kernel takes over: the number of threads, how much of a row they hold, rows in
pieces, rows in turns, rows longer than what is held, each with rows that start on a line and rows that do not.  Against the
64-bit formulas on a few rows (the bounds are those of test_gpu_losses) and against the other ways through on all."""
import numpy as np
import pytest
import torch

import losses_reference as ref
import paper_2203_16340_amd as L
from gpu_helpers import DEV
from test_gpu_losses import HALF_UNIT, dev, host, labels_of, logits_of, near_grad, near_values

pytestmark = pytest.mark.gpu

# chunks of 16 bytes in a row: on both sides of 64 x 4, 128 x 4, 256 x 4, 256 x 8, 512 x 8, 512 x 10, 512 x 13, 512 x 16, 1024 x 13, 1024 x 16
CHUNKS = [1, 255, 257, 511, 513, 1025, 2049, 4096, 4103, 5121, 6657, 8192, 8199, 13313, 16384, 16391, 20001]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("chunks", CHUNKS)
def test_many_rows_of_every_length(chunks, dtype):
    per = 16 // torch.tensor([], dtype=dtype).element_size()
    rows = 66                                          # more than are split
    for extra in (0, 3):                               # rows on chunks; rows on any element
        vocab = chunks * per + extra
        z = logits_of(rows, vocab, dtype, seed=chunks).to(DEV)
        y = labels_of(rows, vocab, seed=chunks, ignored=0.1)
        y[:4] = [0, vocab - 1, vocab // 2, -1]
        yd = dev(y, torch.int64)
        top = min(vocab, 40)
        rng = np.random.default_rng(chunks)
        index = np.stack([rng.choice(vocab, top, replace=False) for _ in range(rows)])
        a = dev(rng.normal(size=(rows, top)) + 3)
        lse = dev(np.logaddexp.reduce(host(a), axis=1) + 0.2)
        adv, old = dev(rng.normal(size=rows)), dev(-5 - rng.random(rows))
        old_np, adv_np = host(old), host(adv)
        picked = [0, 1, 2, 3, rows - 1]                # rows that the 64-bit formulas are worked out for
        zs = host(z[picked])
        ones = np.ones(len(picked))

        p = L.policy_loss(z, yd, old, adv, clip_low=1.0, clip_high=1e9)
        want = ref.policy(zs, y[picked], old_np[picked], adv_np[picked], None, ones, 1.0, 1.0, 1e9, 0.0, "k3", 0.0, 1.0)
        ratio = 1 + np.exp(want[2] - old_np[picked]).max() * np.abs(adv_np).max()
        near_values(p.logp[picked], want[2])
        near_values(p.row_loss[picked], want[1], 2 * ratio)
        near_grad(p.grad[picked], want[4], ratio)
        e = L.policy_loss(z, yd, old, adv, clip_low=1.0, clip_high=1e9, entropy_coef=0.3, entropy=True)
        want = ref.policy(zs, y[picked], old_np[picked], adv_np[picked], None, ones, 1.0, 1.0, 1e9, 0.0, "k3", 0.3, 1.0)
        near_values(e.entropy[picked], want[3])
        near_grad(e.grad[picked], want[4], ratio + 1)

        for given in (None, lse):
            d = L.distill_loss(z, torch.as_tensor(index).to(DEV), a, teacher_lse=given)
            want = ref.distill(zs, index[picked], host(a)[picked], None if given is None else host(given)[picked], ones, 1.0, 1.0)
            near_values(d.row_loss[picked], want[1], 12)
            near_grad(d.grad[picked], want[2], 1.0)
            # every row of the gradient sums to nothing, away from rounding: sum_j p_j = sum_j q_j (with the rest, where there is one)
            if given is None or vocab > top:
                off = d.grad.double().sum(1).abs()
                assert off.max() <= 1e-4 + HALF_UNIT[dtype] * 2.2

        t = L.token_logprob(z, yd, entropy=True)
        assert torch.allclose(t.logp, p.logp, rtol=1e-5, atol=2e-5) and torch.allclose(t.entropy, e.entropy, rtol=1e-5, atol=4e-5)
        # the same rows, few enough to be split, and without a gradient
        few = slice(0, 64)
        q = L.policy_loss(z[few], yd[few], old[few], adv[few], clip_low=1.0, clip_high=1e9)
        assert torch.allclose(q.grad.float(), p.grad[few].float(), rtol=2.2 * HALF_UNIT[dtype] + 2e-5, atol=4e-5 * ratio)
        n = L.policy_loss(z, yd, old, adv, clip_low=1.0, clip_high=1e9, grad=False)
        assert torch.allclose(n.row_loss, p.row_loss, rtol=1e-5, atol=4e-5 * ratio)
        # the gradient in the logits' place is the same gradient
        for make in (lambda x, g: L.policy_loss(x, yd, old, adv, clip_low=1.0, clip_high=1e9, grad=g).grad,
                     lambda x, g: L.distill_loss(x, torch.as_tensor(index).to(DEV), a, teacher_lse=lse, grad=g).grad,
                     lambda x, g: L.token_logprob_grad(x, yd, t, adv, grad=g)):
            here = z.clone()
            assert torch.equal(make(here, here), make(z, True))


@pytest.mark.parametrize("vocab", [66000, 131072, 140001])
def test_more_rows_than_workgroups_take_turns(vocab):
    """1500 rows for 512 workgroups, some not counted, against the same rows a few at a time."""
    rows = 1500
    g = torch.Generator(device=DEV).manual_seed(3)
    z = torch.randn(rows, vocab, device=DEV, generator=g).to(torch.bfloat16)
    y = torch.randint(0, vocab, (rows,), device=DEV, generator=g)
    w = (torch.rand(rows, device=DEV, generator=g) > 0.3).float()
    w[rows - 600:rows - 550] = 0
    old = torch.full((rows,), -12.0, device=DEV)
    adv = torch.randn(rows, device=DEV, generator=g)
    p = L.policy_loss(z, y, old, adv, weight=w)
    total = 0.0
    for at in range(0, rows, 60):
        part = slice(at, min(at + 60, rows))
        q = L.policy_loss(z[part], y[part], old[part], adv[part], weight=w[part])
        assert torch.allclose(q.row_loss, p.row_loss[part], rtol=1e-4, atol=1e-4)
        assert torch.allclose(q.grad.float(), p.grad[part].float(), rtol=0.01, atol=1e-6)
        total += q.loss.double().item()
    assert abs(p.loss.item() - total) <= 1e-4 * p.row_loss.abs().sum().item()
    assert (p.grad[w == 0] == 0).all() and (p.grad[w != 0].abs().amax(1) > 0).float().mean() > 0.3


def test_label_in_every_place_of_a_row():
    """The label's entry is written apart from its chunk: first and last single element, first and last of a chunk, every slot."""
    for vocab, shift in ((4103, 1), (66003, 3), (140003, 5)):
        at = torch.tensor([0, 1, 2, 6, 7, 8, 9, 511, 512, 4095, 4096, 4097, 4102, vocab // 3, vocab // 2, vocab - 9, vocab - 8, vocab - 7, vocab - 2,
                           vocab - 1], device=DEV)
        room = torch.zeros(len(at) * 4, vocab + 13, dtype=torch.bfloat16, device=DEV)
        z = room[:, shift:shift + vocab]                # (a uniform distribution: all other entries are alike)
        y = at.repeat(4)
        old = torch.full((len(y),), -float(np.log(vocab)), device=DEV)
        one = torch.ones(len(y), device=DEV)
        t = L.token_logprob(z, y)
        for grad in (L.policy_loss(z, y, old, one).grad, L.token_logprob_grad(z, y, t, -one)):
            rest = grad.clone()
            rest[torch.arange(len(y), device=DEV), y] = 0
            mine = grad[torch.arange(len(y), device=DEV), y].float()
            assert torch.allclose(mine, torch.full_like(mine, -1.0), rtol=0.01)
            assert torch.allclose(rest.float().sum(1), torch.ones_like(mine), rtol=0.01) and (torch.count_nonzero(rest, 1) == vocab - 1).all()


def test_the_widest_vocabulary_of_the_distillation():
    """2^19 entries, 1024 of them the teacher's: the largest LDS; whole rows and rows in pieces."""
    vocab, top = 1 << 19, 1024
    z = logits_of(66, vocab, torch.bfloat16, seed=2).to(DEV)
    rng = np.random.default_rng(5)
    index = torch.as_tensor(np.stack([rng.choice(vocab, top, replace=False) for _ in range(66)])).to(DEV)
    a = dev(rng.normal(size=(66, top)) + 6)
    lse = torch.logsumexp(a, 1) + 0.2
    for rows in (66, 3):
        for given in (None, lse[:rows].contiguous()):
            d = L.distill_loss(z[:rows], index[:rows], a[:rows], teacher_lse=given)
            want = ref.distill(host(z[:2]), index[:2].cpu().numpy(), host(a[:2]), None if given is None else host(given[:2]), np.ones(2), 1.0, 1.0)
            near_values(d.row_loss[:2], want[1], 12)
            near_grad(d.grad[:2], want[2], 1.0)
    with pytest.raises(L.LbfgsbError):
        L.distill_loss(torch.zeros(1, vocab + 1, device=DEV), index[:1], a[:1])


def test_rows_in_pieces_recorded_into_a_graph():
    rows, vocab = 8, 70001
    z = logits_of(rows, vocab, torch.bfloat16).to(DEV)
    y = dev(labels_of(rows, vocab), torch.int64)
    old, adv = torch.full((rows,), -9.0, device=DEV), torch.linspace(-1, 1, rows, device=DEV)
    index, a = torch.randint(0, vocab, (rows, 16), device=DEV), torch.randn(rows, 16, device=DEV)

    def step():
        t, p, d = L.token_logprob(z, y, entropy=True), L.policy_loss(z, y, old, adv), L.distill_loss(z, index, a)
        return [t.logp, t.lse, t.entropy, p.loss, p.row_loss, p.grad, d.loss, d.row_loss, d.grad]

    step()
    st = torch.cuda.Stream(device=DEV)
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        out = step()
    for k in range(3):
        z.copy_(logits_of(rows, vocab, torch.bfloat16, seed=30 + k))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for g, want in zip(got, step()):
            assert torch.equal(g, want)
        torch.cuda.synchronize()
