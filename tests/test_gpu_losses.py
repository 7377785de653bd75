"""The losses on logits through the library, against the 64-bit formulas of losses_reference.

Bounds, from the arithmetic (eps = 2^-24, half a unit of 32 bits):
  * an exponential's argument (z - m) s has two roundings, so a term is off by 2 eps |argument| + the instruction's unit, where a
    term that counts has an argument of at most ~40: 1e-5 of it.  Averaged over a distribution the arguments are at
    most ~25, and sums run over at most ~100 dependent additions: ln S is off by at most 25 * 2 eps + 100 eps < 1e-5.
    A value (logp, lse, H, a loss) may be off by 2e-5 (its own and the entropy's sum), plus 4 eps of its size for its rounding.
  * a gradient is W (p - ...): off by 1e-5 of each term's size and 2e-5 W where terms cancel, rounded once to the type.
  * policy: the ratio exp(logp - old) and the KL term take logp's error times their slope (at most 20 here).
"""
import numpy as np
import pytest
import torch

import losses_reference as ref
import paper_2203_16340_amd as L
from gpu_helpers import DEV

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
HALF_UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
SMALLEST = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
SHAPES = [(1, 1), (1, 2), (3, 7), (5, 64), (2, 511), (3, 4096), (4, 4097), (130, 1000), (2, 50021), (1, 131073), (3, 262147)]


def near_values(got, want, slope=1.0):
    got = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    want = np.asarray(want)
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want)), (got, want)
    both = ~np.isnan(want)
    inf = np.isinf(want) & both
    assert np.array_equal(got[inf], want[inf])
    fine = both & ~inf
    off = np.abs(got[fine] - want[fine]) - (2e-5 * slope + 4 * EPS * np.abs(want[fine]))
    assert off.size == 0 or off.max() <= 0, (off.max(), got[fine][off.argmax()], want[fine][off.argmax()])


def near_grad(got, want, size):
    """size: the largest weight of a row's gradient, times the slope"""
    t = got.dtype
    got = got.double().cpu().numpy()
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    bound = (HALF_UNIT[t] * 1.01 + 1e-5) * np.abs(want[fine]) + 2e-5 * size + SMALLEST[t]
    off = np.abs(got[fine] - want[fine]) - bound
    assert off.max() <= 0, (off.max(), got[fine][off.argmax()], want[fine][off.argmax()])


def logits_of(rows, vocab, dtype, seed=0, spread=3.0):
    g = torch.Generator().manual_seed(seed + rows * 1000003 + vocab)
    return (torch.randn(rows, vocab, generator=g) * spread).to(dtype)


def host(z):
    return z.double().cpu().numpy()


def labels_of(rows, vocab, seed=0, ignored=0.0):
    rng = np.random.default_rng(seed + rows + vocab)
    y = rng.integers(0, vocab, rows)
    y[rng.random(rows) < ignored] = -100
    return y


def dev(a, dtype=torch.float32):
    return torch.as_tensor(np.ascontiguousarray(a)).to(DEV, dtype)


# ---- token log-probabilities ---------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_token_logprob_and_its_gradient(rows, vocab, dtype):
    z, y = logits_of(rows, vocab, dtype), labels_of(rows, vocab, ignored=0.2 if rows > 4 else 0.0)
    for temperature in (1.0, 0.6):
        s = 1 / temperature
        zd, yd = z.to(DEV), dev(y, torch.int64)
        r = L.token_logprob(zd, yd, temperature=temperature, entropy=True)
        want = ref.token_logprob(host(z), y, s)
        for got, w in zip((r.logp, r.lse, r.entropy), want):
            near_values(got, w)
        near_values(r.lse.double() + r.lse_rest.double(), want[1])
        plain = L.token_logprob(zd, yd, temperature=temperature)
        assert plain.entropy is None and torch.equal(plain.logp, r.logp) and torch.equal(plain.lse, r.lse)
        rng = np.random.default_rng(7)
        d, e = rng.normal(size=rows), rng.normal(size=rows)
        d32, e32 = dev(d), dev(e)
        d, e = host(d32), host(e32)
        got = L.token_logprob_grad(zd, yd, r, d32, temperature=temperature)
        near_grad(got, ref.token_grad(host(z), y, s, d), s * np.abs(d).max())
        got = L.token_logprob_grad(zd, yd, r, d32, temperature=temperature, d_entropy=e32)
        # (the entropy's term: log p_j + H is at most ~40, each of its parts off by 2e-5)
        near_grad(got, ref.token_grad(host(z), y, s, d, e), s * (np.abs(d).max() + 3 * np.abs(e).max()))


def _masked_rows(dtype, vocab):
    """Rows whose masks are as bad as masks get."""
    low = torch.finfo(dtype).min
    z = logits_of(8, vocab, dtype, seed=5)
    z[0, 1:] = -torch.inf            # one entry left
    z[1, :] = -torch.inf             # none
    z[2, 1:] = low                   # one, masked by the lowest value
    z[3, :] = low                    # all alike: a uniform row
    z[4, vocab // 2:] = -torch.inf
    z[5, ::2] = low
    z[6, 0] = torch.finfo(dtype).max
    z[7, :-1] = -torch.inf           # the last entry alone
    y = np.array([0, 1, 0, vocab - 1, 0, 1, 0, vocab - 1])
    return z, y


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [9, 1030, 40001])
def test_masked_rows(dtype, vocab):
    z, y = _masked_rows(dtype, vocab)
    zd, yd = z.to(DEV), dev(y, torch.int64)
    r = L.token_logprob(zd, yd, entropy=True)
    want = ref.token_logprob(host(z), y, 1.0)
    for got, w in zip((r.logp, r.lse, r.entropy), want):
        near_values(got, w)
    one = torch.ones(8, device=DEV)
    g = L.token_logprob_grad(zd, yd, r, one, d_entropy=one)
    near_grad(g, ref.token_grad(host(z), y, 1.0, np.ones(8), np.ones(8)), 4.0)
    z32 = host(z)
    old = np.where(np.isfinite(want[0]), want[0], -3.0) - 0.05
    p = L.policy_loss(zd, yd, dev(old), one, entropy_coef=0.1, entropy=True)
    w = ref.policy(z32, y, host(dev(old)), np.ones(8), None, np.ones(8), 1.0, 0.2, 0.2, 0.0, "k3", 0.1, 1.0)
    near_values(p.logp, w[2])
    near_values(p.row_loss, w[1], slope=2)
    near_grad(p.grad, w[4], 4.0)


def test_rows_that_do_not_count_are_not_read_and_bad_ones_stay_alone():
    vocab = 3001
    z = logits_of(6, vocab, torch.float32)
    z[0, 5] = torch.nan              # ignored row
    z[1, 7] = torch.nan              # a row that counts
    z[2, 3] = torch.inf
    y = np.array([-1, 2, 4, vocab, 0, 1])            # row 3: a label past the vocabulary
    zd, yd = z.to(DEV), dev(y, torch.int64)
    r = L.token_logprob(zd, yd, entropy=True)
    lp = r.logp.cpu().numpy()
    assert lp[0] == 0 and r.lse[0] == 0 and r.entropy[0] == 0
    assert np.isnan(lp[1]) and np.isnan(lp[2]) and np.isnan(lp[3]) and np.isfinite(lp[4:]).all()
    w = torch.tensor([1.0, 1, 1, 1, 0, 1], device=DEV)
    old = torch.full((6,), -3.0, device=DEV)
    for p in (L.policy_loss(zd, yd, old, torch.ones(6, device=DEV), weight=w, entropy=True),):
        g = p.grad.cpu().numpy()
        assert (g[0] == 0).all() and (g[4] == 0).all() and np.isfinite(g[5]).all() and p.row_loss[4] == 0
        assert np.isnan(g[1]).any() and np.isnan(g[2]).any() and np.isnan(g[3]).all()
        assert torch.isnan(p.loss)
    g = L.token_logprob_grad(zd, yd, r, torch.ones(6, device=DEV)).cpu().numpy()
    assert (g[0] == 0).all() and np.isnan(g[3]).all() and np.isfinite(g[4:]).all()
    # the rows that are fine are what they are without the others
    alone = L.token_logprob(zd[4:].contiguous(), yd[4:].contiguous())
    assert torch.equal(alone.logp, r.logp[4:])


# ---- policy ----------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
@pytest.mark.parametrize("kl_kind,entropy_coef", [(None, 0.0), ("k1", 0.0), ("k2", 0.03), ("k3", 0.0)])
def test_policy_loss(rows, vocab, dtype, kl_kind, entropy_coef):
    z, y = logits_of(rows, vocab, dtype, seed=1, spread=2.0), labels_of(rows, vocab, seed=1, ignored=0.2 if rows > 4 else 0.0)
    s = 1 / 0.9
    rng = np.random.default_rng(rows * vocab)
    logp = ref.token_logprob(host(z), y, s)[0]
    x = 0.3 * rng.normal(size=rows)
    for edge in (np.log(1.25), np.log(0.8)):         # none on an edge, where either gradient is right
        x[np.abs(x - edge) < 1e-3] = edge + 4e-3
    old, r = dev(logp - x), dev(logp - 0.3 * rng.normal(size=rows))
    adv, w = dev(rng.normal(size=rows)), dev(rng.random(rows) + 0.1)
    if rows > 4:
        w[2] = 0
    kl_coef = 0.0 if kl_kind is None else 0.2
    p = L.policy_loss(z.to(DEV), dev(y, torch.int64), old, adv, ref_logp=r if kl_kind else None, weight=w, clip_low=0.2, clip_high=0.25,
                      kl_coef=kl_coef, kl_kind=kl_kind or "k3", entropy_coef=entropy_coef, temperature=0.9, scale=2.0, entropy=True)
    total, loss, lp, H, grad = ref.policy(host(z), y, host(old), host(adv), host(r), host(w), s, 0.2, 0.25, kl_coef, kl_kind or "k3",
                                          entropy_coef, 2.0)
    near_values(p.logp, lp)
    near_values(p.entropy, H)
    slope = 1 + 2 * np.abs(host(adv)).max()
    near_values(p.row_loss, loss, slope)
    near_values(p.loss, total, slope * 2 * host(w).sum())
    near_grad(p.grad, grad, 2 * s * host(w).max() * slope)
    none = L.policy_loss(z.to(DEV), dev(y, torch.int64), old, adv, ref_logp=r if kl_kind else None, weight=w, clip_low=0.2, clip_high=0.25,
                         kl_coef=kl_coef, kl_kind=kl_kind or "k3", entropy_coef=entropy_coef, temperature=0.9, scale=2.0, grad=False)
    assert none.grad is None and none.entropy is None
    near_values(none.loss, total, slope * 2 * host(w).sum())


def test_policy_ratio_held_on_the_right_side():
    """Four tokens: ratio above and below the range, advantage of either sign; two have a gradient, two have none."""
    z = torch.zeros(4, 8, device=DEV)
    lp = -np.log(8.0)
    x = np.array([0.5, 0.5, -0.5, -0.5])
    adv = np.array([1.0, -1.0, 1.0, -1.0])
    p = L.policy_loss(z, torch.zeros(4, dtype=torch.int64, device=DEV), dev(lp - x), dev(adv))
    near_values(p.row_loss, np.array([-1.2, np.exp(0.5), -np.exp(-0.5), 0.8]), 2)
    g = p.grad.cpu().numpy()
    assert (g[0] == 0).all() and (g[3] == 0).all() and (g[1:3, 0] != 0).all()


# ---- distillation ----------------------------------------------------------------------------------------------------------


def _teacher(rows, vocab, top, seed, index_type, padded):
    rng = np.random.default_rng(seed)
    index = np.stack([rng.permutation(vocab)[:top] if vocab <= 5000 else rng.choice(vocab, top, replace=False) for _ in range(rows)])
    a = rng.normal(size=(rows, top)) * 2 + 4
    if padded:
        for r in range(rows):
            n = rng.integers(0, top + 1)
            index[r, n:] = -1
        a[rows // 2, top // 2] = -np.inf
    return index.astype(np.int32 if index_type == torch.int32 else np.int64), a


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (2, 7, 7), (3, 64, 5), (2, 511, 65), (40, 1000, 200), (3, 4097, 1024), (2, 50021, 64),
                                            (2, 131073, 33), (1, 262147, 128)])
def test_distill_loss(rows, vocab, top, rest, dtype):
    s = 0.5
    for padded, index_type in ((False, torch.int64), (True, torch.int32)):
        z = logits_of(rows, vocab, dtype, seed=2)
        index, a = _teacher(rows, vocab, top, vocab + top, index_type, padded)
        ad = dev(a)
        a = host(ad)
        rng = np.random.default_rng(3)
        w = dev(rng.random(rows) + 0.1)
        if rows > 4:
            w[1] = 0
        lse = None
        if rest:
            scaled = np.where(index >= 0, a * s, -np.inf)
            lse = dev(np.where(np.isfinite(scaled).any(1), np.logaddexp.reduce(scaled, axis=1), 1.0) + 0.3)
        r = L.distill_loss(z.to(DEV), torch.as_tensor(index).to(DEV), ad, teacher_lse=lse, temperature=2.0, weight=w, scale=3.0)
        total, loss, grad = ref.distill(host(z), index, a, None if lse is None else host(lse), host(w), s, 3.0)
        # (log q and log p are off by 1e-5 each, and q by as much of itself, under logarithms of at most ~20)
        near_values(r.row_loss, loss, 12)
        near_values(r.loss, total, 12 * 3 * host(w).sum())
        near_grad(r.grad, grad, 3 * s * host(w).max())
        assert L.distill_loss(z.to(DEV), torch.as_tensor(index).to(DEV), ad, teacher_lse=lse, temperature=2.0, weight=w, scale=3.0,
                              grad=False).grad is None


@pytest.mark.parametrize("rest", [False, True])
def test_distill_index_that_comes_twice_and_student_masks(rest):
    vocab = 700
    z = logits_of(6, vocab, torch.float32, seed=9)
    z[1, 400:] = -torch.inf
    z[2, :] = -torch.inf
    z[3, 20:] = torch.finfo(torch.float32).min
    index = np.tile(np.array([5, 9, 5, 11, 9, 5, 300]), (6, 1))
    index[3] = [0, 3, 3, 7, -1, 12, 19]
    index[5] = [1, 1, 1, 1, 1, 1, 1]
    a = np.random.default_rng(0).normal(size=(6, 7)) + 2
    a[4, 1] = -np.inf
    ad = dev(a)
    a = host(ad)
    lse = dev(np.logaddexp.reduce(a, axis=1) + 0.5) if rest else None
    w = np.ones(6)
    r = L.distill_loss(z.to(DEV), torch.as_tensor(index).to(DEV), ad, teacher_lse=lse)
    total, loss, grad = ref.distill(host(z), index, a, None if lse is None else host(lse), w, 1.0, 1.0)
    near_values(r.row_loss, loss, 12)
    near_grad(r.grad, grad, 1.0)


def test_distill_teacher_types_padding_and_index_past_the_vocabulary():
    z = logits_of(3, 100, torch.bfloat16, seed=4)
    index = np.array([[1, 2, 100], [3, -5, -1], [-1, -1, -1]])
    a = np.array([[1.0, 2.0, 3.0], [2.0, np.nan, np.inf], [np.nan, 1.0, 1.0]])     # whatever stands in the padding
    r = L.distill_loss(z.to(DEV), torch.as_tensor(index).to(DEV), dev(a))
    assert torch.isnan(r.row_loss[0]) and torch.isnan(r.grad[0]).all()
    assert torch.isfinite(r.row_loss[1:]).all() and torch.isfinite(r.grad[1:].float()).all()
    assert r.row_loss[2] == 0 and (r.grad[2] == 0).all()
    rng = np.random.default_rng(1)
    a = rng.normal(size=(3, 4))
    index = np.array([[1, 2, 50, 9]] * 3)
    for t in (torch.bfloat16, torch.float16):
        at = dev(a, t)
        r = L.distill_loss(z.to(DEV), torch.as_tensor(index).to(DEV), at)
        total, loss, grad = ref.distill(host(z), index, host(at), None, np.ones(3), 1.0, 1.0)
        near_values(r.row_loss, loss, 12)
        near_grad(r.grad, grad, 1.0)


def test_distill_against_a_student_that_agrees():
    """Student and teacher alike: no loss and no gradient, with the rest's outcome as well."""
    z = logits_of(4, 5000, torch.float32, seed=6)
    index = torch.topk(z, 50, dim=1).indices
    a = z.gather(1, index)
    r = L.distill_loss(z.to(DEV), index.to(DEV), a.to(DEV), teacher_lse=torch.logsumexp(z.double(), 1).float().to(DEV))
    assert r.row_loss.abs().max() < 5e-5 and r.grad.abs().max() < 2e-5


# ---- preference ------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("kind", ["sigmoid", "hinge", "ipo"])
@pytest.mark.parametrize("normalised", [False, True])
@pytest.mark.parametrize("pairs,longest", [(1, 1), (1, 3000), (3, 17), (70, 130)])
def test_preference_loss(kind, normalised, pairs, longest):
    rng = np.random.default_rng(pairs * longest)
    lengths = rng.integers(0, longest + 1, 2 * pairs)
    off = 3 + np.concatenate([[0], np.cumsum(lengths)])
    T = int(off[-1]) + 4                              # tokens before the first answer and after the last belong to none
    logp, r = dev(-2 * rng.random(T)), dev(-2 * rng.random(T))
    mask = torch.as_tensor(rng.random(T) < 0.8).to(DEV)
    logp[~mask] = torch.nan                           # what does not count may hold anything
    w = dev(rng.random(pairs) + 0.1)
    for reference, m in ((r, mask), (None, mask), (r, None)):
        lp = logp if m is not None else torch.nan_to_num(logp, nan=-1.0)
        smoothing = 0.1 if kind == "sigmoid" else 0.0
        got = L.preference_loss(lp, reference, dev(off, torch.int64), mask=m, weight=w, beta=0.3, kind=kind, label_smoothing=smoothing,
                                margin=0.2, length_normalised=normalised, scale=2.0)
        clean = np.nan_to_num(host(lp))
        total, losses, R, grad = ref.preference(clean, None if reference is None else host(r), off, None if m is None else m.cpu().numpy(),
                                                host(w), 0.3, kind, smoothing, 0.2, normalised, 2.0)
        # everything is in 64 bits up to the rounding of the results
        for g, want in ((got.loss, total), (got.pair_loss, losses), (got.rewards, R), (got.grad, grad)):
            want = np.asarray(want)
            g = host(g)
            assert np.abs(g - want).max() <= 2 * EPS * np.abs(want).max() + 1e-12
        assert torch.equal(L.preference_loss(lp, reference, dev(off, torch.int64), mask=m, weight=w, beta=0.3, kind=kind,
                                             label_smoothing=smoothing, margin=0.2, length_normalised=normalised, scale=2.0,
                                             grad=False).loss, got.loss)


def test_preference_offsets_are_taken_into_the_tokens():
    lp = torch.full((10,), -1.0, device=DEV)
    off = torch.tensor([-4, 3, 99], dtype=torch.int64, device=DEV)
    r = L.preference_loss(lp, None, off, beta=1.0)
    assert r.rewards.tolist() == [-3.0, -7.0]
    off = torch.tensor([8, 5, 12], dtype=torch.int64, device=DEV)      # does not ascend: the first answer is empty
    r = L.preference_loss(lp, None, off, beta=1.0)
    assert r.rewards.tolist() == [0.0, -5.0]


def test_a_pair_of_weight_zero_does_not_count():
    lp = torch.tensor([-1.0, -torch.inf, -1.0, -2.0], device=DEV)
    off = torch.arange(5, dtype=torch.int64, device=DEV)
    r = L.preference_loss(lp, None, off, weight=torch.tensor([1.0, 0.0], device=DEV))
    assert torch.isfinite(r.loss) and r.grad[1] == 0 and r.grad[3] == 0 and (r.grad[[0, 2]] != 0).all()


def test_no_rows_no_tokens_no_pairs():
    z = torch.empty(0, 50, device=DEV)
    y, f = torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV)
    assert L.token_logprob(z, y, entropy=True).logp.shape == (0,)
    assert L.token_logprob_grad(z, y, L.token_logprob(z, y), f).shape == (0, 50)
    p = L.policy_loss(z, y, f, f)
    assert p.loss == 0 and p.grad.shape == (0, 50)
    assert L.distill_loss(z, torch.empty(0, 4, dtype=torch.int64, device=DEV), torch.empty(0, 4, device=DEV)).loss == 0
    r = L.preference_loss(torch.ones(3, device=DEV), None, torch.zeros(1, dtype=torch.int64, device=DEV))
    assert r.loss == 0 and (r.grad == 0).all() and r.rewards.shape == (0,)
    r = L.preference_loss(f, None, torch.zeros(3, dtype=torch.int64, device=DEV))
    assert abs(r.loss.item() - np.log(2)) < 1e-6 and r.grad.shape == (0,)


# ---- layouts, streams, graphs ------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("first,vocab,ld", [(0, 4096, 4104), (1, 1001, 1003), (3, 4099, 4107), (5, 70001, 70013)])
def test_rows_on_any_element_and_gradients_elsewhere(first, vocab, ld, dtype):
    rows = 5
    big = logits_of(rows, ld, dtype, seed=8).to(DEV)
    z = big[:, first:first + vocab]
    y = dev(labels_of(rows, vocab), torch.int64)
    flat = z.contiguous()
    one = torch.ones(rows, device=DEV)
    old = -torch.arange(rows, device=DEV).float()
    index = torch.arange(0, 60, 6, device=DEV).repeat(rows, 1)
    a = torch.arange(10.0, device=DEV).repeat(rows, 1)
    room = torch.full((rows, ld + 9), 7.0, dtype=dtype, device=DEV)
    out = room[:, 2:2 + vocab]
    t, tf = L.token_logprob(z, y, entropy=True), L.token_logprob(flat, y, entropy=True)
    for got, want in zip((t.logp, t.lse, t.entropy), (tf.logp, tf.lse, tf.entropy)):
        assert torch.allclose(got, want, rtol=1e-6, atol=1e-5)        # (sums over other pieces)
    for make in (lambda q, g: L.token_logprob_grad(q, y, tf, one, d_entropy=one, grad=g),
                 lambda q, g: L.policy_loss(q, y, old, one, grad=g, entropy_coef=0.1).grad,
                 lambda q, g: L.distill_loss(q, index, a, grad=g).grad,
                 lambda q, g: L.distill_loss(q, index, a, grad=g, teacher_lse=torch.logsumexp(a, 1) + 0.1).grad):
        want = make(flat, True).float()
        room.fill_(7.0)
        got = make(z, out)
        assert got.data_ptr() == out.data_ptr()
        size = want.abs().max().item()
        assert torch.allclose(got.float(), want, rtol=2.1 * HALF_UNIT[dtype] + 2e-5, atol=2e-5 * max(1.0, size))
        assert (room[:, :2] == 7).all() and (room[:, 2 + vocab:] == 7).all()      # nothing beside the gradient is written
        here = big.clone()[:, first:first + vocab]
        assert torch.equal(make(here, here), got)                       # in place
        mine = flat.clone()
        assert torch.equal(make(mine, mine), make(flat, True))
    assert torch.equal(big, logits_of(rows, ld, dtype, seed=8).to(DEV))


def test_rows_far_apart_pass_32_bit_offsets():
    ld = (1 << 30) + 24
    big = torch.zeros(3 * ld, dtype=torch.bfloat16, device=DEV)
    z = big.as_strided((3, 5000), (ld, 1))
    z.copy_(logits_of(3, 5000, torch.bfloat16))
    y = torch.tensor([1, 4999, 3], device=DEV)
    flat = z.contiguous()
    r, rf = L.token_logprob(z, y), L.token_logprob(flat, y)
    assert torch.equal(r.logp, rf.logp)
    one = torch.ones(3, device=DEV)
    g = L.policy_loss(flat, y, r.logp, one).grad
    assert torch.equal(L.token_logprob_grad(z, y, r, one), L.token_logprob_grad(flat, y, r, one))
    assert torch.equal(L.policy_loss(z, y, r.logp, one, grad=z).grad, g)
    assert torch.count_nonzero(big) == torch.count_nonzero(g)


def test_same_bits_on_another_stream_and_from_call_to_call():
    z = logits_of(300, 33001, torch.bfloat16).to(DEV)
    y = dev(labels_of(300, 33001), torch.int64)
    old = -torch.ones(300, device=DEV)
    first = L.policy_loss(z, y, old, old, entropy=True)
    st = torch.cuda.Stream(device=DEV)
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        second = L.policy_loss(z, y, old, old, entropy=True)
    torch.cuda.current_stream().wait_stream(st)
    third = L.policy_loss(z, y, old, old, entropy=True)
    for a, b, c in zip(first, second, third):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_recorded_into_a_graph():
    rows, vocab = 40, 20011
    z = logits_of(rows, vocab, torch.bfloat16).to(DEV)
    y = dev(labels_of(rows, vocab), torch.int64)
    off = torch.tensor([0, 9, 20, 28, 40], dtype=torch.int64, device=DEV)
    index = torch.randint(0, vocab, (rows, 16), device=DEV)
    a = torch.randn(rows, 16, device=DEV)

    def step():
        t = L.token_logprob(z, y, entropy=True)
        p = L.preference_loss(t.logp, None, off)
        g = L.token_logprob_grad(z, y, t, p.grad)
        q = L.policy_loss(z, y, t.logp, t.logp)
        d = L.distill_loss(z, index, a)
        return [*t, p.loss, p.grad, g, q.loss, q.grad, d.loss, d.grad]

    step()
    st = torch.cuda.Stream(device=DEV)
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        out = step()
    for k in range(3):
        z.copy_(logits_of(rows, vocab, torch.bfloat16, seed=20 + k))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for g, want in zip(got, step()):
            assert torch.equal(g, want)
        torch.cuda.synchronize()


# ---- refusals ------------------------------------------------------------------------------------------------------------------


def test_refusals():
    z = torch.zeros(4, 10, device=DEV)
    y = torch.zeros(4, dtype=torch.int64, device=DEV)
    f = torch.zeros(4, device=DEV)
    t = L.token_logprob(z, y)
    idx, a = torch.zeros(4, 3, dtype=torch.int64, device=DEV), torch.zeros(4, 3, device=DEV)
    with pytest.raises(TypeError):
        L.token_logprob(z.double(), y)
    with pytest.raises(TypeError):
        L.token_logprob(z.t(), torch.zeros(10, dtype=torch.int64, device=DEV))
    with pytest.raises(TypeError):
        L.token_logprob(z.cpu(), y)
    with pytest.raises(TypeError):
        L.token_logprob(z, y.int())
    with pytest.raises(ValueError):
        L.token_logprob(z, y[:3].contiguous())
    with pytest.raises(L.LbfgsbError):
        L.token_logprob(z[:1].expand(4, 10), y)                    # rows that lie on each other
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(L.LbfgsbError):
            L.token_logprob(z, y, temperature=bad)
    with pytest.raises(L.LbfgsbError):
        L.token_logprob_grad(z, y, t, f, d_entropy=f)              # needs the entropy
    with pytest.raises(TypeError):
        L.token_logprob_grad(z, y, t, f, grad=False)
    with pytest.raises(TypeError):
        L.token_logprob_grad(z, y, t, f, grad=z.bfloat16())
    both = torch.zeros(9, 10, device=DEV)
    with pytest.raises(L.LbfgsbError) as e:
        L.policy_loss(both[:4], y, f, f, grad=both[2:6])           # half over the logits
    assert "overlap" in str(e.value)
    with pytest.raises(L.LbfgsbError):
        L.policy_loss(z, y, f, f, kl_coef=0.1)                     # no reference
    with pytest.raises(ValueError):
        L.policy_loss(z, y, f, f, kl_kind="k4")
    with pytest.raises(L.LbfgsbError):
        L.policy_loss(z, y, f, f, clip_low=1.5)
    with pytest.raises(L.LbfgsbError):
        L.policy_loss(z, y, f, f, scale=float("inf"))
    with pytest.raises(TypeError):
        L.policy_loss(z, y, f.double(), f)
    with pytest.raises(ValueError):
        L.distill_loss(z, idx, a[:, :2])
    with pytest.raises(TypeError):
        L.distill_loss(z, idx.short(), a)
    with pytest.raises(L.LbfgsbError):
        L.distill_loss(z, torch.zeros(4, 1025, dtype=torch.int64, device=DEV), torch.zeros(4, 1025, device=DEV))
    with pytest.raises(ValueError):
        L.preference_loss(f, None, torch.zeros(4, dtype=torch.int64, device=DEV))
    off = torch.zeros(3, dtype=torch.int64, device=DEV)
    for kw in (dict(beta=0.0), dict(label_smoothing=1.0), dict(kind="hinge", label_smoothing=0.1), dict(margin=float("nan"))):
        with pytest.raises(L.LbfgsbError):
            L.preference_loss(f, None, off, **kw)
    with pytest.raises(ValueError):
        L.preference_loss(f, None, off, kind="logistic")
