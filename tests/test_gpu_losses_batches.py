"""The losses on logits over batches of many long rows of 16 bits, where two workgroups share a compute unit and hold a row in registers, or
in registers and LDS: against the same rows a few hundred at a time, which go another way, and against softmaxes in 64 bits."""
import pytest
import torch

import paper_2203_16340_amd as L
from gpu_helpers import DEV
from test_gpu_losses import HALF_UNIT

pytestmark = pytest.mark.gpu

WEIGHT = 64.0            # lifts gradients of f16 out of its subnormal numbers
PART = 200               # rows at a time of the other way: more than are cut in pieces, fewer than are taken in pairs


def room_for(rows, vocab, dtype, on_lines, seed):
    """Rows on lines, or on any element with gaps between them."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    shift, ld = (0, vocab) if on_lines else (3, vocab + 13)
    room = torch.empty(rows, ld, dtype=dtype, device=DEV)
    z = room[:, shift:shift + vocab]
    for at in range(0, rows, PART):
        z[at:at + PART] = (3 * torch.randn(min(PART, rows - at), vocab, device=DEV, generator=g)).to(dtype)
    return z, g


def near(got, want, p, dtype):
    """Both are roundings of one number that is known to 2e-5 of itself, and to 2e-5 of its probability where it is a difference
    of shares."""
    assert torch.equal(got.isnan(), want.isnan())
    bound = (2.02 * HALF_UNIT[dtype] + 2e-5) * want.double().abs() + 2e-5 * WEIGHT * p + (2.0 ** -24 if dtype == torch.float16 else 0.0)
    off = (got.double() - want.double()).abs() - bound
    assert not (off[~want.isnan()] > 0).any()


def probabilities(z):
    return torch.softmax(z.double(), 1).nan_to_num(0.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,vocab,on_lines", [(257, 65537, False), (300, 94208, True), (300, 94152, False), (1500, 94153, False), (1499, 94300, False),
                                                 (1501, 100003, False), (1500, 131072, True), (1503, 134000, False), (1500, 136000, False)])
def test_policy_over_many_long_rows(rows, vocab, on_lines, dtype):
    z, g = room_for(rows, vocab, dtype, on_lines, 5)
    z[7, 5:9] = -torch.inf
    z[8] = -torch.inf
    z[9, vocab // 2] = torch.nan
    y = torch.randint(0, vocab, (rows,), device=DEV, generator=g)
    y[:6] = torch.tensor([0, vocab - 1, vocab // 2, -1, 1, vocab - 2], device=DEV)
    w = torch.where(torch.rand(rows, device=DEV, generator=g) > 0.1, WEIGHT, 0.0)
    w[:10] = WEIGHT
    lse = torch.cat([torch.logsumexp(z[at:at + PART].double(), 1) for at in range(0, rows, PART)])
    old = (z[torch.arange(rows, device=DEV), y.clamp(min=0)].double() - lse).float().nan_to_num(-9.0, posinf=-9.0, neginf=-9.0)
    adv = torch.rand(rows, device=DEV, generator=g) - 0.5

    def loss(part, grad=True):
        return L.policy_loss(z[part], y[part], old[part], adv[part], weight=w[part], grad=grad)

    all_rows = slice(0, rows)
    p = loss(all_rows)
    for at in range(0, rows, PART):
        part = slice(at, min(at + PART, rows))
        q = loss(part)
        assert torch.allclose(q.row_loss, p.row_loss[part], rtol=1e-5, atol=4e-5 * WEIGHT, equal_nan=True)
        near(p.grad[part], q.grad, probabilities(z[part]), dtype)
    assert (p.grad[3] == 0).all() and (p.grad[w == 0] == 0).all()
    again = loss(all_rows)
    assert torch.equal(p.grad.view(torch.int16), again.grad.view(torch.int16))
    here = loss(all_rows, z)                              # (the gradient in the logits' place; the last use of z)
    assert torch.equal(p.grad.view(torch.int16), here.grad.view(torch.int16))


@pytest.mark.parametrize("rows,vocab,top,rest", [(257, 65537, 40, False), (300, 94152, 1024, False), (1500, 94153, 64, False), (1500, 100003, 1024, False),
                                                 (1501, 120000, 16, False), (1500, 131072, 64, False), (4001, 65601, 40, True), (4000, 94000, 1024, True),
                                                 (4000, 94300, 16, True)])
def test_distillation_over_many_long_rows(rows, vocab, top, rest):
    dtype = torch.bfloat16
    z, g = room_for(rows, vocab, dtype, False, 6)
    z[7, 5:9] = -torch.inf
    z[9, vocab // 2] = torch.nan
    w = torch.where(torch.rand(rows, device=DEV, generator=g) > 0.1, WEIGHT, 0.0)
    w[:10] = WEIGHT
    index = torch.randint(0, vocab, (rows, top), device=DEV, generator=g)
    index[0, 1] = index[0, 0]
    index[1, 0], index[1, 1], index[2, 3], index[4] = 0, vocab - 1, -1, -1
    a = torch.randn(rows, top, device=DEV, generator=g) + 3
    lse = torch.logsumexp(a, 1) + 0.4 if rest else None

    def loss(part, grad=True):
        return L.distill_loss(z[part], index[part], a[part], teacher_lse=lse[part] if rest else None, weight=w[part], grad=grad)

    all_rows = slice(0, rows)
    d = loss(all_rows)
    for at in range(0, rows, PART):
        part = slice(at, min(at + PART, rows))
        q = loss(part)
        assert torch.allclose(q.row_loss, d.row_loss[part], rtol=1e-5, atol=4e-5, equal_nan=True)
        near(d.grad[part], q.grad, probabilities(z[part]), dtype)
    assert (d.grad[w == 0] == 0).all()
    # (from the formula: away from the entries dz = w (p - 0), and with the rest w p (1 - r / t))
    picked = torch.tensor([5, 6, rows - 1], device=DEV)
    p = probabilities(z[picked])
    mark = torch.zeros_like(p, dtype=torch.bool).scatter_(1, index[picked], True)
    if rest:
        r = 1 - torch.exp(a[picked].double() - lse[picked, None].double()).sum(1, keepdim=True)
        want = p * (1 - r / p.masked_fill(mark, 0).sum(1, keepdim=True))
    else:
        want = p
    want = (want * w[picked, None].double()).masked_fill(mark, 0)
    near(d.grad[picked].masked_fill(mark, 0), want, p, dtype)
    assert torch.equal(d.grad.view(torch.int16), loss(all_rows).grad.view(torch.int16))
    here = loss(all_rows, z)                              # (the gradient in the logits' place; the last use of z)
    assert torch.equal(d.grad.view(torch.int16), here.grad.view(torch.int16))
