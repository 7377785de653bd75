"""Products with 4-bit weights through the library, against the 64-bit definition.

Bound, from the arithmetic: codes, and x in one or (32 bits) three bf16 parts, are exact in the matrix instructions, so what is lost is
lost in sums in 32 bits: at most 3 * group additions to a group's two sums, then two multiply-adds a group and the sum over up to
8 waves.  With a unit of 2^-23 for an addition whose rounding the hardware may choose, y is off by
(3 * group + 3 * groups + 8) 2^-23 * sum |scale| (code + |zero|) |x|, and then by half a unit of its type.  That counts every addition as if the whole
sum stood there, so the same difference is held to the root of the count, 8 times over, on inputs of random signs as well."""
import numpy as np
import pytest
import torch

import paper_2203_16340_amd as L
import rollouts_reference as ref
from gpu_helpers import DEV

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def plain(rows, cols, group, scale_type, zero, seed=0):
    rng = np.random.default_rng(seed + 7 * rows + cols)
    codes = rng.integers(0, 256, (rows, -(-cols // 2)), dtype=np.uint8)
    groups = -(-cols // group)
    scale = torch.from_numpy(0.02 * (0.3 + rng.random((rows, groups)))).to(scale_type)
    z = torch.from_numpy(rng.integers(0, 16, (rows, groups)) + rng.choice([0.0, 0.25], (rows, groups))).to(scale_type) if zero else None
    return codes, scale, z


def packed(codes, scale, zero, cols, group):
    return L.pack4(torch.from_numpy(codes).to(DEV), scale.to(DEV), None if zero is None else zero.to(DEV), cols=cols, group=group)


def wide(t):
    return None if t is None else t.double().cpu().numpy()


def check(y, x, codes, scale, zero, cols, group, random=True):
    w = ref.weights(codes, wide(scale), wide(zero), cols, group)
    size = np.abs(ref.weights(codes, wide(scale), np.zeros_like(wide(scale)), cols, group))
    size += np.repeat(np.abs(wide(scale)) * (8.0 if zero is None else np.abs(wide(zero))), group, 1)[:, :cols]
    x = wide(x)
    want, total = x @ w.T, np.abs(x) @ size.T
    groups = -(-cols // group)
    adds = 3 * min(group, cols) + 3 * groups + 8
    half = torch.finfo(y.dtype).eps / 2
    got = wide(y)
    assert got.shape == want.shape and np.isfinite(got).all()
    smallest = 2.0 ** -25 if y.dtype == torch.float16 else 0.0
    off = np.abs(got - want) - half * 1.01 * np.abs(want) - smallest
    assert (off <= adds * 2.0 ** -23 * total).all(), (off / total).max()
    if random:
        assert (off <= 8 * adds ** 0.5 * 2.0 ** -23 * np.sqrt((x ** 2) @ (size ** 2).T + 1e-300)).all()


SHAPES = [(1, 1, 1), (1, 3, 33), (2, 64, 128), (1, 65, 127), (5, 100, 129), (4, 1000, 64), (3, 63, 1000), (16, 130, 257), (17, 70, 300), (33, 200, 512),
          (64, 129, 1031), (1, 4097, 2048), (2, 16385, 640), (7, 16500, 131), (20, 16400, 1100)]


@pytest.mark.parametrize("scale_type", TYPES)
@pytest.mark.parametrize("x_type", TYPES)
@pytest.mark.parametrize("tokens,rows,cols", SHAPES)
def test_products(tokens, rows, cols, x_type, scale_type):
    for group, zero in ((32, True), (64, False), (128, True), (256, False), (32, False), (2048, True)):
        codes, scale, z = plain(rows, cols, group, TYPES[scale_type], zero)
        w = packed(codes, scale, z, cols, group)
        x = torch.randn(tokens, cols, generator=torch.Generator().manual_seed(cols)).to(TYPES[x_type]).to(DEV)
        y = L.matvec4(x, w)
        assert y.dtype == x.dtype
        check(y, x, codes, scale, z, cols, group)
        if x_type != "f32":
            check(L.matvec4(x, w, dtype=torch.float32), x, codes, scale, z, cols, group)


# x in LDS as a whole, at its largest and past it, and laid out beforehand; few rows of weights and many; tiles of x by their number
LONG = [(16, 70, 2560), (16, 70, 2570), (9, 80, 5000), (12, 16390, 2700), (40, 32800, 130), (20, 49200, 130),
        (50, 49200, 130), (70, 49200, 64), (6, 33000, 200), (130, 100, 260)]


@pytest.mark.parametrize("x_type,scale_type", [("f32", "f32"), ("bf16", "f16"), ("f16", "bf16")])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("tokens,rows,cols", LONG)
def test_longer_products(tokens, rows, cols, group, x_type, scale_type):
    codes, scale, z = plain(rows, cols, group, TYPES[scale_type], True)
    w = packed(codes, scale, z, cols, group)
    x = torch.randn(tokens, cols, generator=torch.Generator().manual_seed(cols)).to(TYPES[x_type]).to(DEV)
    check(L.matvec4(x, w, dtype=torch.float32), x, codes, scale, z, cols, group)


def test_every_code_and_column_is_where_it_belongs():
    """x picks one column at a time: y is then that column's weights to the bit."""
    rows, cols, group = 70, 261, 32
    codes, scale, z = plain(rows, cols, group, torch.float32, True)
    w = packed(codes, scale, z, cols, group)
    want = ref.weights(codes, wide(scale), wide(z), cols, group)
    eye = torch.eye(cols, device=DEV)
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        got = L.matvec4(eye.to(dtype), w, dtype=torch.float32)
        # (scale times an exact difference of a code and a zero: one rounding, or two where the zero's product was rounded)
        assert np.abs(wide(got).T - want).max() <= 2.0 ** -22 * np.abs(want).max()


@pytest.mark.parametrize("dtype", TYPES)
def test_small_and_large_numbers(dtype):
    rows, cols, group = 65, 200, 64
    codes, scale, z = plain(rows, cols, group, torch.float32, True)
    w = packed(codes, scale, z, cols, group)
    top = {"f32": 1e36, "bf16": 1e36, "f16": 60000.0}[dtype]
    # (the third part of a 32-bit number has 2^-16 of its size: numbers of 2^-100 keep all three)
    low = {"f32": 2.0 ** -90, "bf16": 2.0 ** -110, "f16": 2.0 ** -24}[dtype]
    x = torch.randn(3, cols, generator=torch.Generator().manual_seed(3))
    x = torch.stack([x[0].clamp(-1, 1) * top, (x[1] * 4).round() * low, x[2]]).to(TYPES[dtype]).to(DEV)
    y = L.matvec4(x, w, dtype=torch.float32)
    check(y[:1] / top, x[:1].double() / top, codes, scale, z, cols, group)
    check(y[1:2].double() / low, x[1:2].double() / low, codes, scale, z, cols, group) if dtype != "f32" else None
    check(y[2:], x[2:], codes, scale, z, cols, group)
    if dtype == "f32":
        want = wide(x[1:2]) @ ref.weights(codes, wide(scale), wide(z), cols, group).T
        assert np.abs(wide(y[1:2]) - want).max() <= 2.0 ** -18 * np.abs(want).max()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_finite_stays_in_its_row(dtype, bad):
    codes, scale, z = plain(130, 300, 128, torch.float16, True)
    w = packed(codes, scale, z, 300, 128)
    x = torch.randn(6, 300, generator=torch.Generator().manual_seed(1)).to(TYPES[dtype]).to(DEV)
    x[2, 299] = bad
    y = L.matvec4(x, w)
    assert not torch.isfinite(y[2]).any()
    keep = [0, 1, 3, 4, 5]
    check(y[keep], x[keep], codes, scale, z, 300, 128)


def test_strides_and_a_result_in_place():
    codes, scale, z = plain(97, 161, 32, torch.bfloat16, False)
    w = packed(codes, scale, z, 161, 32)
    for dtype in TYPES.values():
        store = torch.full((5, 400), float("nan"), dtype=dtype, device=DEV)
        x = store[:, 3:164]
        x.copy_(torch.randn(5, 161, generator=torch.Generator().manual_seed(2)))
        want = L.matvec4(x.contiguous(), w)
        assert torch.equal(L.matvec4(x, w), want)
        out = torch.full((5, 301), 7.0, dtype=dtype, device=DEV)
        view = out[:, 5:102]
        before = view._version
        got = L.matvec4(x, w, out=view)
        assert got.data_ptr() == view.data_ptr() and view._version > before
        assert torch.equal(view, want) and (out[:, :5] == 7).all() and (out[:, 102:] == 7).all()
        wider = torch.empty(5, 97, device=DEV)
        L.matvec4(x, w, out=wider)
        assert torch.equal(wider, L.matvec4(x, w, dtype=torch.float32))
    assert L.matvec4(x[:0], w).shape == (0, 97)


def test_tokens_come_alone_as_they_come_together():
    """A row's result does not depend on what stands beside it."""
    codes, scale, z = plain(300, 700, 64, torch.float32, True)
    w = packed(codes, scale, z, 700, 64)
    x = torch.randn(70, 700, device=DEV, generator=torch.Generator(DEV).manual_seed(4)).bfloat16()
    y = L.matvec4(x, w)
    for i in (0, 3, 15, 16, 47, 69):
        check(y[i:i + 1], x[i:i + 1], codes, scale, z, 700, 64)
        assert torch.equal(L.matvec4(x[i:i + 1], w), L.matvec4(x[i:i + 1], w))


@pytest.mark.parametrize("symmetric", [False, True])
@pytest.mark.parametrize("scale_type", TYPES)
@pytest.mark.parametrize("w_type", TYPES)
def test_quantising(w_type, scale_type, symmetric):
    rows, cols, group = 37, 197, 64
    w = torch.randn(rows, cols, generator=torch.Generator().manual_seed(5))
    w[3] = 0.0
    w[4] = w[4].abs()
    w[5, 64:128] = -w[5, 64:128].abs()
    w = w.to(TYPES[w_type])
    store = torch.zeros(rows, 300, dtype=w.dtype, device=DEV)
    store[:, 1:198] = w.to(DEV)
    got = L.quantize4(store[:, 1:198], group=group, symmetric=symmetric, scale_dtype=TYPES[scale_type])
    assert got.scale.dtype == TYPES[scale_type] and (got.zero is None) == symmetric
    # the definition's steps in 32 bits, as they are rounded; a code on the border between two may be either's
    f = np.float32
    q, scale, zero = ref.quantized(w.double().numpy(), group, symmetric, lambda s: float(torch.tensor(float(f(s))).to(TYPES[scale_type])))
    assert np.allclose(wide(got.scale), scale, rtol=torch.finfo(TYPES[scale_type]).eps, atol=0)
    if not symmetric:
        assert np.array_equal(wide(got.zero), zero)
    have = wide(got.scale)
    codes = got.codes.cpu().numpy()
    mine = np.stack([codes & 15, codes >> 4], 2).reshape(rows, -1)
    assert (mine[:, cols:] == 0).all()
    mine = mine[:, :cols]
    at = np.repeat(have, group, 1)[:, :cols]
    exact = np.divide(w.double().numpy(), at, out=np.zeros_like(at), where=at > 0) + np.repeat(zero, group, 1)[:, :cols]
    assert (np.abs(mine - np.clip(exact, 0, 15)) <= 0.5 + 1e-4).all()
    pack = L.pack4(*got, cols=cols, group=group)
    x = torch.randn(2, cols, device=DEV, generator=torch.Generator(DEV).manual_seed(6))
    check(L.matvec4(x, pack), x, codes, got.scale, got.zero, cols, group)


def test_weights_that_are_not_finite():
    w = torch.randn(4, 128, device=DEV)
    w[1, 70], w[2, 3] = float("nan"), float("inf")
    for symmetric in (False, True):
        q = L.quantize4(w, group=64, symmetric=symmetric)
        assert torch.equal(torch.isfinite(q.scale), torch.tensor([[1, 1], [1, 0], [0, 1], [1, 1]], device=DEV).bool())
        y = L.matvec4(torch.ones(1, 128, device=DEV), L.pack4(*q, group=64))
        assert torch.equal(torch.isfinite(y[0]), torch.tensor([1, 0, 0, 1], device=DEV).bool())


def test_refusals():
    codes, scale, z = plain(64, 128, 64, torch.float32, True)
    c, s, z = torch.from_numpy(codes).to(DEV), scale.to(DEV), z.to(DEV)
    for bad in (lambda: L.pack4(c, s[:, :1], group=64), lambda: L.pack4(c, s, z[:10], group=64), lambda: L.pack4(c, s, z, cols=200, group=64)):
        with pytest.raises((TypeError, ValueError)):
            bad()
    for bad in (lambda: L.pack4(c.int(), s, group=64), lambda: L.pack4(c, s.double(), group=64), lambda: L.pack4(c, s, z.half(), group=64),
                lambda: L.pack4(c[:, ::2], s, group=64, cols=64)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(L.LbfgsbError):
        L.pack4(c, s, group=48)
    with pytest.raises(L.LbfgsbError):
        L.quantize4(torch.zeros(4, 64, device=DEV), group=31)
    w = L.pack4(c, s, z, group=64)
    assert "64 x 128" in repr(w)
    x = torch.zeros(2, 128, device=DEV)
    with pytest.raises(ValueError):
        L.matvec4(x[:, :127], w)
    for bad in (lambda: L.matvec4(x.double(), w), lambda: L.matvec4(x.t(), w), lambda: L.matvec4(x, w, dtype=torch.float16), lambda: L.matvec4(x, w, dtype=7),
                lambda: L.matvec4(x, w, out=torch.zeros(2, 63, device=DEV)), lambda: L.matvec4(x, w, out=torch.zeros(2, 64)),
                lambda: L.matvec4(x, w, dtype=torch.float32, out=torch.zeros(2, 64, device=DEV).half())):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(L.LbfgsbError):
        L.matvec4(x, w, out=torch.zeros(2, 64, device=DEV).half())
    with pytest.raises(L.LbfgsbError):
        store = torch.zeros(2, 128, device=DEV)
        L.matvec4(store, w, out=store[:, :64])


def test_history_inference_mode_and_a_result_that_was_kept():
    codes, scale, z = plain(200, 256, 64, torch.float32, True)
    w = packed(codes, scale, z, 256, 64)
    x = torch.randn(20, 256, device=DEV, generator=torch.Generator(DEV).manual_seed(9))
    want = L.matvec4(x, w)
    assert not L.matvec4(x.clone().requires_grad_(), w).requires_grad
    with torch.inference_mode():
        out = torch.empty(20, 200, device=DEV)
        assert torch.equal(L.matvec4(x, w, out=out), want)
    # a way back that kept the tensor which is written over is refused, as after any operation in place
    leaf = torch.ones(20, 200, device=DEV, requires_grad=True)
    kept = torch.tanh(leaf)
    loss = kept.sum()
    L.matvec4(x, w, out=kept.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_calls_on_two_streams_at_once():
    """With a workspace each: x is laid out there."""
    codes, scale, z = plain(3000, 512, 128, torch.float16, True)
    w = packed(codes, scale, z, 512, 128)
    xs = [torch.randn(40, 512, device=DEV, generator=torch.Generator(DEV).manual_seed(k)).half() for k in range(2)]
    want = [L.matvec4(x, w) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for k, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[k].append(L.matvec4(xs[k], w))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[k]) for k in range(2) for g in got[k])


@pytest.mark.parametrize("tokens", [17, 40, 64])
def test_a_replayed_graph_of_more_rows(tokens):
    codes, scale, z = plain(500, 300, 32, torch.bfloat16, False)
    w = packed(codes, scale, z, 300, 32)
    x = torch.zeros(tokens, 300, device=DEV, dtype=torch.bfloat16)
    L.matvec4(x, w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = L.matvec4(x, w)
    for seed in range(4):
        x.copy_(torch.randn(tokens, 300, device=DEV, generator=torch.Generator(DEV).manual_seed(seed)))
        graph.replay()
        want = L.matvec4(x, w)
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_a_replayed_graph_and_another_stream():
    codes, scale, z = plain(1000, 512, 128, torch.float16, True)
    w = packed(codes, scale, z, 512, 128)
    x = torch.randn(3, 512, device=DEV, generator=torch.Generator(DEV).manual_seed(8)).half()
    out = torch.empty(3, 1000, dtype=torch.float16, device=DEV)
    L.matvec4(x, w, out=out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.matvec4(x, w, out=out)
    for seed in range(4):
        x.copy_(torch.randn(3, 512, device=DEV, generator=torch.Generator(DEV).manual_seed(20 + seed)))
        graph.replay()
        want = L.matvec4(x, w)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    with torch.cuda.stream(side):
        got = L.matvec4(x, w)
    side.synchronize()
    assert torch.equal(got, want)
