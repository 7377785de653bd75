"""Products with 4-bit weights in every way that a call is cut into workgroups, waves and tiles: by the rows of x, by how long they are, by the rows of W, by
the types of x and of the scales and by the group.  Against the definition in 64 bits, with the bounds of test_gpu_weights4."""
import pytest
import torch

import paper_2203_16340_amd as L
from gpu_helpers import DEV

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def weights_on_the_gpu(rows, cols, group, scale_type, zero):
    g = torch.Generator(DEV).manual_seed(rows + 7 * cols)
    groups = -(-cols // group)
    codes = torch.randint(0, 256, (rows, -(-cols // 2)), device=DEV, dtype=torch.uint8, generator=g)
    scale = (0.02 * (0.3 + torch.rand(rows, groups, device=DEV, generator=g))).to(scale_type)
    z = (torch.randint(0, 16, (rows, groups), device=DEV, generator=g) + 0.25 * torch.randint(0, 2, (rows, groups), device=DEV, generator=g)).to(scale_type) if zero else None
    return codes, scale, z


def check_in_parts(y, x, codes, scale, zero, cols, group):
    """the bounds of test_gpu_weights4.check, some rows of W at a time"""
    at = torch.arange(cols, device=DEV) // group
    adds = 3 * min(group, cols) + 3 * scale.shape[1] + 8
    half = torch.finfo(y.dtype).eps / 2
    x = x.double()
    step = max(64, (1 << 26) // cols)
    assert torch.isfinite(y).all()
    for r in range(0, len(codes), step):
        part = codes[r:r + step]
        code = torch.stack([part & 15, part >> 4], 2).view(len(part), -1)[:, :cols].double()
        s = scale[r:r + step].double()[:, at]
        z = 8.0 if zero is None else zero[r:r + step].double()[:, at]
        want = x @ (s * (code - z)).t()
        size = s * (code + (z if zero is None else z.abs()))
        del code, s, z
        off = (y[:, r:r + step].double() - want).abs() - half * 1.01 * want.abs()
        assert (off <= adds * 2.0 ** -23 * (x.abs() @ size.t())).all()
        assert (off <= 8 * adds ** 0.5 * 2.0 ** -23 * ((x ** 2) @ (size ** 2).t()).sqrt()).all()


def product(tokens, rows, cols, group, x_type, scale_type, zero):
    codes, scale, z = weights_on_the_gpu(rows, cols, group, TYPES[scale_type], zero)
    w = L.pack4(codes, scale, z, cols=cols, group=group)
    x = torch.randn(tokens, cols, device=DEV, generator=torch.Generator(DEV).manual_seed(cols)).to(TYPES[x_type])
    y = L.matvec4(x, w, dtype=torch.float32)
    check_in_parts(y, x, codes, scale, z, cols, group)
    assert torch.equal(L.matvec4(x, w, dtype=torch.float32), y)


# blocks of 64 rows of W: below 256, from there, from 512, from 768
FEW = [(1, 1000, 300), (16, 1000, 300), (16, 1000, 2700), (1, 16400, 300), (1, 32800, 300), (2, 32800, 300), (16, 16400, 300), (16, 32800, 300), (16, 16400, 2700),
       (16, 32800, 2700)]
MORE = [(20, 1000, 300), (40, 1000, 300), (60, 1000, 300), (20, 32800, 200), (20, 49200, 200), (40, 16400, 200), (40, 32800, 200), (40, 49200, 200), (60, 32800, 200),
        (60, 49200, 200), (140, 32800, 130)]


@pytest.mark.parametrize("scale_type", TYPES)
@pytest.mark.parametrize("x_type", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("tokens,rows,cols", FEW + MORE)
def test_plans(tokens, rows, cols, group, x_type, scale_type):
    product(tokens, rows, cols, group, x_type, scale_type, tokens % 3 != 0)


# one row of x that takes more than half of the room for it in LDS, and all of it
@pytest.mark.parametrize("group,scale_type", [(32, "f32"), (64, "f16"), (128, "bf16"), (4096, "f32")])
@pytest.mark.parametrize("x_type,rows,cols", [("f32", 32800, 6900), ("f32", 16400, 13700), ("f32", 32800, 13700), ("bf16", 32800, 20600), ("f16", 16400, 41100),
                                              ("bf16", 32800, 41100), ("f32", 500, 13700), ("f16", 500, 41100)])
def test_one_long_row(x_type, rows, cols, group, scale_type):
    product(1, rows, cols, group, x_type, scale_type, True)
