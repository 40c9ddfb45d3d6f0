"""Dropout with the residual sum against its definition in 64 bits."""
import pytest
import torch

import paper_1511_06416_amd as same
from tests import cross_reference as ref

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def matrix(rows, cols, dtype, seed=0, stride=None, offset=0):
    g = torch.Generator().manual_seed(seed)
    buf = torch.randn(rows * (stride or cols) + offset, generator=g).to(dtype).cuda()[offset:]
    return buf.view(rows, stride or cols)[:, :cols]


def expect(x, residual, drop, seed, call_id):
    """Value and bound: one product and one sum in fp32, one rounding."""
    x64 = x.cpu().double()
    f = ref.dropout_keep(*x.shape, drop, seed, call_id) if drop else torch.ones_like(x64)
    y = torch.where(f > 0, x64 * f, 0.0) + (0 if residual is None else residual.cpu().double())
    # fp32: the scale's and the sum's roundings (2^-24 each of x f, 2^-24 of y)
    bound = 2.0 ** -24 * (2 * (x64 * f).abs() + 2 * y.abs())
    if x.dtype != torch.float32:
        bound = bound + ref.U[x.dtype] * (y.abs() + bound) + ref.TINY[x.dtype]
    return y, bound


SHAPES = [(1, 1), (1, 7), (1, 8), (3, 5), (257, 330), (64, 1024), (1000, 33), (5, 2049)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("with_residual", [False, True])
@pytest.mark.parametrize("drop", [0.0, 0.1])
def test_values(rows, cols, dtype, with_residual, drop):
    x = matrix(rows, cols, dtype, 1)
    r = matrix(rows, cols, dtype, 2) if with_residual else None
    y = torch.full_like(x, float("nan"))
    same.same_dropout(x, y, drop, 2 ** 63 + 12345, 6, residual=r)
    ref.check("y", y, *expect(x, r, drop, 2 ** 63 + 12345, 6))


@pytest.mark.parametrize("cols,stride,offset", [(33, 40, 0), (64, 72, 0), (64, 72, 1), (24, 24, 3), (24, 25, 0)])
@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_alignment_do_not_change_the_mask(cols, stride, offset, dtype):
    x, r = matrix(50, cols, dtype, 1, stride, offset), matrix(50, cols, dtype, 2, stride + 8, offset)
    y = matrix(50, cols, dtype, 3, stride)
    want = torch.empty((50, cols), dtype=dtype, device="cuda")
    same.same_dropout(x.contiguous().clone(), want, 0.25, 5, 1, residual=r.contiguous().clone())
    before = y._base.clone() if y._base is not None else None
    same.same_dropout(x, y, 0.25, 5, 1, residual=r)
    assert torch.equal(y, want)
    if before is not None and stride > cols:   # what lies between the rows is left alone
        after = y._base.view(50, stride)
        assert torch.equal(after[:, cols:], before.view(50, stride)[:, cols:])


@pytest.mark.parametrize("dtype", TYPES)
def test_in_place_and_beside(dtype):
    x, r = matrix(40, 64, dtype, 1), matrix(40, 64, dtype, 2)
    want = torch.empty_like(x)
    same.same_dropout(x, want, 0.5, 9, 0, residual=r)
    a, b = x.clone(), r.clone()
    same.same_dropout(a, a, 0.5, 9, 0, residual=r)
    same.same_dropout(x, b, 0.5, 9, 0, residual=b)
    assert torch.equal(a, want) and torch.equal(b, want)
    wide = torch.zeros(40, 128, dtype=dtype, device="cuda")   # two column blocks of one buffer
    wide[:, :64] = x
    same.same_dropout(wide[:, :64], wide[:, 64:], 0.5, 9, 0, residual=r)
    assert torch.equal(wide[:, 64:], want)


def test_gradient():
    """The gradient is the same call without the residual: against the
    formula's, and against differences, exact for a linear map."""
    x, dy = matrix(100, 37, torch.float32, 1), matrix(100, 37, torch.float32, 2)
    dx = torch.empty_like(x)
    same.same_dropout(dy, dx, 0.25, 77, 2)
    ref.check("dx", dx, *expect(dy, None, 0.25, 77, 2))
    y, y2 = torch.empty_like(x), torch.empty_like(x)
    same.same_dropout(x, y, 0.25, 77, 2)
    same.same_dropout(x + 1.0, y2, 0.25, 77, 2)
    diff = ((y2 - y).double() * dy.double()).cpu()
    # the difference's own roundings: x + 1, both scalings
    allowed = 2.0 ** -21 * (x.abs().cpu().double() + 2) * dy.abs().cpu().double() * 2
    assert bool(((diff - dx.cpu().double()).abs() <= allowed).all())


def test_share_and_independence():
    n = 1 << 20
    x = torch.ones(1, n, device="cuda")
    ys = []
    for seed, call in ((1, 0), (1, 1), (2, 0)):
        y = torch.empty_like(x)
        same.same_dropout(x, y, 0.1, seed, call)
        ys.append(y > 0)
        t = round(0.1 * 65536) / 65536
        assert abs(float((y == 0).double().mean()) - t) < 6 * (t * (1 - t) / n) ** 0.5
    for a in range(3):
        for b in range(a):
            both = float((~ys[a] & ~ys[b]).double().mean())
            assert abs(both - 0.01) < 6 * (0.01 / n) ** 0.5


def test_dropped_elements_do_not_use_x():
    x = torch.full((4, 1000), float("nan"), device="cuda")
    r = torch.ones_like(x)
    y = torch.empty_like(x)
    same.same_dropout(x, y, 0.5, 3, 0, residual=r)
    keep = ref.dropout_keep(4, 1000, 0.5, 3, 0) > 0
    assert torch.equal(y.isnan().cpu(), keep) and bool((y.cpu()[~keep] == 1).all())


def test_large_and_on_a_stream():
    """Elements past 2^31: the last ones against the first rows' definition."""
    rows, cols = (1 << 31) // 1024 + 3, 1024
    x = torch.ones(rows, cols, dtype=torch.float16, device="cuda")
    y = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        same.same_dropout(x, y, 0.25, 4, 9)
    side.synchronize()
    first = (rows - 2) * cols
    groups = torch.arange(first // 8, first // 8 + 2 * cols // 8).numpy().astype("uint64")
    w = ref.philox(groups & 0xFFFFFFFF, groups >> 32, 4 << 24, 9, 4)
    half = [((w >> s) & 0xFFFF) for s in (0, 16)]
    import numpy as np
    half = np.stack(half, axis=-1).reshape(2, cols)
    assert torch.equal((y[rows - 2:] > 0).cpu(), torch.from_numpy(half >= 16384))


def test_refusals():
    x = matrix(8, 16, torch.float32)
    y = torch.zeros_like(x)

    def refuse(code, x=x, y=y, drop=0.1, residual=None):
        with pytest.raises(same.SameError) as e:
            same.same_dropout(x, y, drop, 0, 0, residual=residual)
        assert e.value.code == code and str(e.value)

    for drop in (-0.1, 1.0, 1e-6, 1 - 1e-6, float("nan")):
        refuse(same.SAME_EINVAL, drop=drop)
    refuse(same.SAME_EINVAL, y=y.half())
    refuse(same.SAME_EINVAL, y=y[:7])
    refuse(same.SAME_EINVAL, x=x.double(), y=y.double())
    refuse(same.SAME_EINVAL, x=x.cpu())
    refuse(same.SAME_EINVAL, residual=x[:, :8])
    refuse(same.SAME_EINVAL, x=x.T.contiguous().T)
    buf = torch.zeros(9, 16, device="cuda")
    refuse(same.SAME_EINVAL, x=buf[:8], y=buf[1:])
    refuse(same.SAME_EINVAL, x=x, y=buf[:8], residual=buf[1:])
    refuse(same.SAME_EINVAL, y=y[:1].expand(8, 16))
    torch.cuda.synchronize()
    assert not y.any()
    e = torch.empty(0, 16, device="cuda")
    same.same_dropout(e, torch.empty_like(e), 0.1, 0, 0)   # nothing to do
