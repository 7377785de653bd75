"""Packed 4-bit weights that are too short for the sizes they come with, or no bytes in a row, are refused before anything else is looked at."""
import ctypes as C

import pytest
import torch

import paper_2203_16340_amd as L
from paper_2203_16340_amd import losses
from paper_2203_16340_amd import rollouts as R

ROWS, COLS, GROUP, F32, F16 = 100, 300, 64, 1, 3


def need(rows=ROWS, cols=COLS, group=GROUP, scale_type=F16, zero=True):
    return L.lib().lbfgsb_packed4_bytes(C.byref(R.Weights4Struct(rows, cols, group, scale_type, 16, 16, 16 if zero else None)))


def call(packed, rows=ROWS, cols=COLS, group=GROUP, scale_type=F16, zero=True):
    return losses._load().matvec4(torch.zeros(2, cols), packed, rows, cols, group, scale_type, zero, None, None, 0)


def test_whole_weights_come_as_far_as_x():
    for more in (0, 5):
        with pytest.raises(TypeError, match="x must be"):                     # (which is on the host here)
            call(torch.zeros(need() + more, dtype=torch.uint8))


@pytest.mark.parametrize("short", [1, 16, 8192, None])
def test_too_few_bytes(short):
    packed = torch.zeros(need() - short if short else 0, dtype=torch.uint8)
    with pytest.raises(ValueError, match=f"must have {need()} bytes"):
        call(packed)


@pytest.mark.parametrize("other", [dict(rows=129), dict(cols=385), dict(group=32), dict(scale_type=F32), dict(rows=1 << 20)], ids=str)
def test_sizes_that_need_more(other):
    assert need(**other) > need()
    with pytest.raises(ValueError, match="bytes"):
        call(torch.zeros(need(), dtype=torch.uint8), **other)
    with pytest.raises(ValueError, match="bytes"):
        call(torch.zeros(need(zero=False), dtype=torch.uint8))                # (zeros that are not there)


def test_what_is_no_bytes_in_a_row():
    for packed in (torch.zeros(need(), dtype=torch.float32), torch.zeros(2 * need(), dtype=torch.uint8)[::2],
                   torch.zeros(1, dtype=torch.uint8).expand(need()), torch.zeros(need(), dtype=torch.int8)):
        with pytest.raises(TypeError, match="packed weights"):
            call(packed)


@pytest.mark.parametrize("bad", [dict(rows=0), dict(rows=-5), dict(cols=0), dict(group=48), dict(scale_type=0)], ids=str)
def test_sizes_of_no_weights(bad):
    at = dict(rows=ROWS, cols=COLS, group=GROUP, scale_type=F16, zero=True)
    at.update(bad)
    rc, _ = losses._load().matvec4(torch.zeros(2, 8), torch.zeros(1 << 20, dtype=torch.uint8), *at.values(), None, None, 0)
    assert rc == L.E_INVALID_ARG and L.lib().lbfgsb_last_error()
