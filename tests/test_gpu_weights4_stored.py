"""Packed 4-bit weights that were stored and come back: whole they give the same products, and what does not hold them is refused."""
import pytest
import torch

import paper_2203_16340_amd as L
from gpu_helpers import DEV
from test_gpu_weights4 import packed, plain

pytestmark = pytest.mark.gpu

ROWS, COLS, GROUP = 130, 300, 64


def weights():
    codes, scale, zero = plain(ROWS, COLS, GROUP, torch.float16, True)
    return packed(codes, scale, zero, COLS, GROUP)


def again(w, bytes_, rows=ROWS, cols=COLS, group=GROUP, scale_type=3, has_zero=True):
    return L.Weights4(bytes_, rows, cols, group, scale_type, has_zero)


@pytest.mark.parametrize("tokens", [1, 20])
def test_stored_weights(tokens):
    w = weights()
    x = torch.randn(tokens, COLS, device=DEV, generator=torch.Generator(DEV).manual_seed(1)).bfloat16()
    want = L.matvec4(x, w)
    stored = w.packed.cpu()
    assert torch.equal(L.matvec4(x, again(w, stored.to(DEV))), want)
    # in front of other bytes
    longer = torch.cat([w.packed, w.packed.new_full((512,), 255)])
    assert torch.equal(L.matvec4(x, again(w, longer)), want)
    assert torch.equal(L.matvec4(x, again(w, longer[:w.packed.numel()])), want)


def test_what_does_not_hold_them():
    w = weights()
    x = torch.zeros(2, COLS, device=DEV)
    longer = torch.zeros(2 * w.packed.numel(), dtype=torch.uint8, device=DEV)
    for bad in (again(w, w.packed[:-1]), again(w, w.packed[:0]), again(w, w.packed, rows=193), again(w, w.packed, group=32),
                again(w, w.packed, scale_type=1)):
        with pytest.raises(ValueError, match="bytes"):
            L.matvec4(x, bad)
    with pytest.raises(ValueError, match="bytes"):
        L.matvec4(torch.zeros(2, 400, device=DEV), again(w, w.packed, cols=400))
    for bad in (again(w, w.packed.view(torch.int8)), again(w, longer[::2]), again(w, w.packed.cpu())):
        with pytest.raises(TypeError):
            L.matvec4(x, bad)
    with pytest.raises(L.LbfgsbError):
        L.matvec4(x, again(w, longer[8:8 + w.packed.numel()]))            # (not on a boundary of 16 bytes)
    with pytest.raises(L.LbfgsbError):
        L.matvec4(x, again(w, w.packed, group=48))
