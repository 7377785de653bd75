"""What products with 4-bit weights keep of x, and that a row's result is its own.

One entry of x at a time, so that nothing but its own product comes out.  A 32-bit entry goes in as three bf16 parts that hold its 24 bits, each
times a code exact, added in 32 bits: the first addition, to 0, is exact, the other two are off by a unit of 2^-23 of the sum each at most (whose rounding
the hardware may choose), for code x and for x alike; the two multiply-adds behind them by 2^-24 of theirs, and the rest adds zeros.  So y is off by at
most (2 * 2 + 1 + 1) 2^-24 scale (code + |zero|) |x|.  Without the third part it would be off by up to 2^-17 scale |code - zero| |x|."""
import numpy as np
import pytest
import torch

import paper_2203_16340_amd as L
import rollouts_reference as ref
from gpu_helpers import DEV
from test_gpu_weights4 import TYPES, check, packed, plain, wide

pytestmark = pytest.mark.gpu

BOUND = 6 * 2.0 ** -24


def full(n, size, seed=0):
    """numbers of all 24 bits, near `size`"""
    rng = np.random.default_rng(seed + n)
    bits = rng.integers(1 << 23, 1 << 24, n) | 1
    return (bits * 2.0 ** -23 * rng.choice([-1.0, 1.0], n) * size).astype(np.float32)


def one_at_a_time(columns, cols, size):
    x = np.zeros((len(columns), cols), dtype=np.float32)
    x[np.arange(len(columns)), columns] = full(len(columns), size)
    return torch.from_numpy(x).to(DEV)


def parts_are_there(rows, cols, group, zero, columns, tokens, size=1.0):
    codes, scale, z = plain(rows, cols, group, torch.float32, zero)
    w = packed(codes, scale, z, cols, group)
    exact = torch.from_numpy(ref.weights(codes, wide(scale), wide(z), cols, group)).to(DEV)
    spread = torch.from_numpy(ref.weights(codes, wide(scale), np.zeros_like(wide(scale)), cols, group)).to(DEV)
    at = torch.arange(cols, device=DEV) // group
    spread += scale.to(DEV).double()[:, at] * (8.0 if z is None else z.to(DEV).double().abs()[:, at])
    for k in range(0, len(columns), tokens):
        pick = columns[k:k + tokens]
        x = one_at_a_time(pick, cols, size)
        got = L.matvec4(x, w).double()
        own = x.double().sum(1)[:, None]
        off = (got - own * exact[:, pick].t()).abs()
        assert (off <= BOUND * own.abs() * spread[:, pick].t()).all(), (pick, (off / (own.abs() * spread[:, pick].t())).max().item() * 2 ** 24)


# x in LDS as a whole, laid out with one tile of 16 rows, with two; few rows of weights, and as many as take the wide kernels
@pytest.mark.parametrize("group,zero", [(32, True), (64, False), (128, True), (32, False)])
@pytest.mark.parametrize("tokens,rows,cols", [(1, 70, 300), (5, 70, 300), (16, 70, 300), (16, 70, 1000), (17, 70, 300), (32, 70, 300), (300, 70, 300)])
def test_every_column_keeps_all_of_32_bits(tokens, rows, cols, group, zero):
    parts_are_there(rows, cols, group, zero, np.arange(cols), tokens)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("tokens,rows,cols", [(1, 16400, 300), (4, 16400, 300), (1, 32800, 300), (7, 32800, 300), (16, 16400, 1000), (16, 32800, 1000),
                                              (32, 49200, 300)])
def test_many_rows_of_weights_keep_all_of_32_bits(tokens, rows, cols, group):
    parts_are_there(rows, cols, group, True, np.random.default_rng(cols).permutation(cols)[:48], tokens)


@pytest.mark.parametrize("size", [2.0 ** -90, 2.0 ** -102, 2.0 ** 100])
def test_small_and_large_numbers_of_all_bits(size):
    """The third part of a number of 2^-102 begins at 2^-120 and ends at 2^-125, with the smallest normal numbers behind it."""
    for tokens in (1, 16, 40):
        parts_are_there(70, 260, 64, True, np.arange(260), tokens, size)


@pytest.mark.parametrize("size", [2.0 ** -90, 2.0 ** 90])
@pytest.mark.parametrize("tokens,cols", [(3, 200), (16, 1000), (40, 200)])
def test_sums_of_small_and_large_numbers(tokens, cols, size):
    codes, scale, z = plain(65, cols, 64, torch.float32, True)
    w = packed(codes, scale, z, cols, 64)
    x = torch.from_numpy(np.stack([full(cols, size, seed) for seed in range(tokens)])).to(DEV)
    check(L.matvec4(x, w).double() / size, x.double() / size, codes, scale, z, cols, 64)


@pytest.mark.parametrize("x_type", TYPES)
@pytest.mark.parametrize("tokens,rows,cols", [(2, 300, 700), (4, 300, 700), (11, 300, 700), (16, 300, 700), (16, 70, 2700), (16, 16400, 2700), (7, 32800, 200),
                                              (30, 300, 700), (45, 300, 700), (64, 300, 700), (70, 300, 700), (40, 49200, 200)])
def test_a_row_is_its_own_whatever_stands_beside_it(tokens, rows, cols, x_type):
    codes, scale, z = plain(rows, cols, 64, torch.float32, True)
    w = packed(codes, scale, z, cols, 64)
    x = torch.randn(tokens, cols, device=DEV, generator=torch.Generator(DEV).manual_seed(4)).to(TYPES[x_type])
    want = L.matvec4(x, w, dtype=torch.float32)
    assert torch.isfinite(want).all()
    for i in sorted({0, 1, tokens // 2, tokens - 1}):
        for other in (0.0, 1000.0, float("nan"), float("inf")):
            beside = torch.full_like(x, other)
            beside[i] = x[i]
            assert torch.equal(L.matvec4(beside, w, dtype=torch.float32)[i], want[i]), (i, other)
