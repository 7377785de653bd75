"""The 64-bit definitions of what makes rollouts, against what they are for; no GPU."""
import numpy as np

import rollouts_reference as ref


def test_a_number_falls_into_its_token():
    z = np.log([0.1, 0.2, 0.3, 0.4])
    for u, want in ((0.0, 0), (0.0999, 0), (0.1001, 1), (0.2999, 1), (0.3001, 2), (0.6001, 3), (0.9999, 3), (1.0, 3), (-1.0, 0), (7.0, 3)):
        j, lp, _ = ref.draw(z, u, 1.0)
        assert j == want and abs(lp - z[want]) < 1e-12 and ref.room(np.exp(z), want, u) >= 0 > ref.room(np.exp(z), (want + 1) % 4, u)
    assert ref.draw(z, np.nan, 1.0)[0] == -1 and ref.draw(np.full(3, -np.inf), 0.5, 1.0)[0] == -1
    assert ref.draw([-np.inf, 0.0, -np.inf], 0.0, 1.0)[0] == 1 and ref.draw([-np.inf, 0.0, -np.inf], 1.0, 1.0)[0] == 1


def test_what_is_emitted_is_distributed_as_the_target():
    """The whole of both numbers' range, in a grid: the first token's frequencies are p, whatever the drafter's q."""
    rng = np.random.default_rng(0)
    z, zq = rng.normal(size=(2, 5)) * 1.5, rng.normal(size=(1, 5)) * 1.5
    p, q = np.exp(ref.log_softmax(z[0], 1.0)), np.exp(ref.log_softmax(zq[0], 1.0))
    grid = (np.arange(60) + 0.5) / 60
    for draft, share in ((zq, q), (None, np.full(5, 0.2))):
        got = np.zeros(5)
        for x in range(5):
            for u in grid:
                for v in grid:
                    got[ref.verify(z, [x], [u], v, 1.0, draft=draft)[0][0]] += share[x] / 3600
        assert np.abs(got - p).max() < 0.02


def test_codes_stand_for_their_numbers():
    codes = np.array([[0x21, 0x0f], [0x80, 0x07]], dtype=np.uint8)
    w = ref.weights(codes, np.array([[0.5], [2.0]]), None, 3, 32)
    assert np.array_equal(w, [[-3.5, -3.0, 3.5], [-16.0, 0.0, -2.0]])
    w = ref.weights(codes, np.array([[0.5], [2.0]]), np.array([[0.0], [1.5]]), 3, 32)
    assert np.array_equal(w, [[0.5, 1.0, 7.5], [-3.0, 13.0, 11.0]])


def test_quantised_codes_are_the_nearest():
    rng = np.random.default_rng(1)
    w = rng.normal(size=(6, 70))
    w[0] = 0.0
    for symmetric in (False, True):
        q, scale, zero = ref.quantized(w, 32, symmetric, lambda s: s)
        back = np.repeat(scale, 32, 1)[:, :70] * (q - np.repeat(zero, 32, 1)[:, :70])
        assert (np.abs(back - w) <= 0.5001 * np.repeat(scale, 32, 1)[:, :70] * (1 if symmetric else 2)).all()
