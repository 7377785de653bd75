"""Draws and verifications of the longest vocabularies, by both ways of taking them, and rows whose mass lies in a tail of equal entries, where every entry's
rounding points the same way."""
import pytest
import torch

import paper_2203_16340_amd as L
from gpu_helpers import DEV
from test_gpu_draws import TYPES, ROOM, check_draw, check_verify, near_logp

pytestmark = pytest.mark.gpu

LONGEST = 1 << 21


def randn(*shape, seed):
    return torch.randn(*shape, device=DEV, generator=torch.Generator(DEV).manual_seed(seed))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(2, LONGEST), (2, LONGEST - 3), (130, LONGEST), (260, LONGEST - 1)])
def test_draws_from_the_longest_rows(rows, vocab, dtype):
    z = torch.empty(rows, vocab, dtype=TYPES[dtype], device=DEV)
    for r in range(0, rows, 32):
        z[r:r + 32] = randn(*z[r:r + 32].shape, seed=r) * 3
    u = torch.rand(rows, device=DEV, generator=torch.Generator(DEV).manual_seed(1))
    got = L.draw_tokens(z, u)
    few = torch.arange(0, rows, max(1, rows // 3), device=DEV)
    check_draw(z[few], u[few], 1.0, L.DrawTokens(got.tokens[few], got.logp[few]))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("requests", [3, 161])
@pytest.mark.parametrize("given", [False, True])
def test_verification_of_the_longest_rows(requests, dtype, given):
    vocab, drafts = LONGEST, 1
    zq = torch.empty(requests, drafts, vocab, dtype=TYPES[dtype], device=DEV)
    z = torch.empty(requests, drafts + 1, vocab, dtype=TYPES[dtype], device=DEV)
    for i in range(requests):
        zq[i] = randn(drafts, vocab, seed=2 * i) * 2
        z[i, :drafts] = zq[i].float() + 0.7 * randn(drafts, vocab, seed=2 * i + 1)
        z[i, drafts] = zq[i, 0].flip(0)
    g = torch.Generator(DEV).manual_seed(3)
    d = L.draw_tokens(zq[:, 0], torch.rand(requests, device=DEV, generator=g))
    x, lq = d.tokens[:, None].contiguous(), d.logp[:, None].contiguous()
    u, v = torch.rand(requests, drafts, device=DEV, generator=g), torch.rand(requests, device=DEV, generator=g)
    u[0], u[1] = 0.0, 1.0 - 2.0 ** -24                  # accepted; refused unless p is as large as q
    got = L.verify_draft(z, x, u, v, draft_logits=zq, draft_logp=lq if given else None)
    few = torch.tensor(sorted({0, 1, 2, requests - 1}), device=DEV)
    check_verify(L.VerifyDraft(*(t[few] for t in got)), z[few], x[few], u[few], v[few], draft=zq[few], draft_logp=lq[few] if given else None)
    assert got.count.min() >= 1 and got.count.max() == 2 and got.count[0] == 2


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [131072, 1 << 19, 1 << 20, 1 << 21])
def test_rows_with_a_tail_of_equal_entries(vocab, dtype):
    """A few entries at the top and all others as far below as makes the two about alike: a running sum is off by what the tail's one value is off by."""
    far = torch.tensor(vocab / 5).log().item()
    depths = [far - 1, far, far + 0.37, far + 1]
    z = torch.stack([torch.full((vocab,), 4.7 - d) for d in depths])
    z[:, 1000:1005] = 4.7
    z = z.to(TYPES[dtype]).to(DEV)
    u = torch.cat([torch.linspace(0.002, 0.998, 100), torch.rand(60, generator=torch.Generator().manual_seed(vocab))]).to(DEV)
    for row in z:
        many = row.expand(len(u), vocab).contiguous()
        p = torch.softmax(row.double(), 0)
        running = p.cumsum(0)
        for rows in (1, 64, len(u)):                     # (split over workgroups, and a workgroup each)
            got = L.draw_tokens(many[:rows], u[:rows])
            at = u[:rows].double() * running[-1]
            assert ((running[got.tokens] - at) >= -ROOM).all() and ((at - running[got.tokens] + p[got.tokens]) >= -ROOM).all()
            near_logp(got.logp.double().cpu().numpy(), p.log()[got.tokens].cpu().numpy())
