"""Norms of queries and keys with the position rotation against their
definition in 64 bits."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_1511_06416_amd as same

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
U = 2.0 ** -24
HALF = {t: torch.finfo(t).eps / 2 for t in TYPES}
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


def angles(rot, base=10_000.0):
    return base ** (-2.0 * np.arange(rot // 2) / max(rot, 1))


def heads(n, h, d, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n, h, d, generator=g) * scale).to(dtype).cuda()


def reference(x, w, pos, a, eps, dy=None):
    """(y, bound) or ((dx, bound), (dw, bound)), on the CPU in 64 bits.

    Bounds: a sum of d <= 128 squares in chains of 16 and exchanges has a
    relative error below 24 U, its root 12 U, the hardware's reciprocal root
    and its Newton step 4 U, x r w 2 U: 18 U, taken as 24.  Cosine and sine are
    off by 4 U at most (the reduced angle's rounding 2^-28 of a turn, the
    series 2^-30, the last rounding), the rotation's sums by 3 U of its terms.
    """
    x, d = x.cpu().double(), x.shape[-1]
    w = torch.ones(d, dtype=torch.float64) if w is None else w.cpu().double()
    h = 0 if a is None else len(a)
    r = (x.square().mean(-1, keepdim=True) + float(np.float32(eps))).rsqrt()
    xhat = x * r
    if h:
        t = pos.cpu().double()[:, None, None] * torch.from_numpy(a)
        c, s = t.cos(), t.sin()

    def turn(z, sign):
        lo, hi, rest = z[..., :h], z[..., h:2 * h], z[..., 2 * h:]
        return torch.cat([lo * c - sign * hi * s, hi * c + sign * lo * s, rest], dim=-1) if h else z

    def size(z):   # of the terms of a rotation
        both = z[..., :h].abs() + z[..., h:2 * h].abs()
        return torch.cat([both, both, z[..., 2 * h:].abs()], dim=-1)

    if dy is None:
        z = xhat * w
        return turn(z, 1.0), 32 * U * size(z)
    dy = dy.cpu().double()
    dz, e = turn(dy, -1.0), 8 * U * size(dy)
    u = dz * w
    m = (u * xhat).mean(-1, keepdim=True)
    dx = r * (u - xhat * m)
    # of m: every term's own error (xhat's 24 U, dz's, a product) and the sum's 24 U
    em = ((u * xhat).abs() * 50 * U + (e * w.abs() * xhat.abs())).mean(-1, keepdim=True)
    bound = r * (e * w.abs() + u.abs() * 26 * U + (xhat * m).abs() * 52 * U + xhat.abs() * em)
    n = x.shape[0] * x.shape[1]
    terms = dz * xhat
    # a sum of n terms in any order: n U of their absolute values
    dw = terms.sum((0, 1)), (terms.abs() * (26 + n) * U + e * xhat.abs()).sum((0, 1))
    return (dx, bound), dw


def check(name, got, want, bound):
    t = got.dtype
    got = got.cpu().double()
    if t != torch.float32:
        bound = bound + HALF[t] * (want.abs() + bound) + TINY[t]
    else:
        bound = bound + U * want.abs()
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), "%s: %d of %d off, first %s: %s for %s" % (
        name, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), got[bad][0], want[bad][0])


SHAPES = [  # q, k, heads of q and k, width, turned
    (501, 77, 1, 1, 64, 64), (300, 1001, 2, 1, 40, 8), (133, 200, 1, 2, 128, 128), (65, 9, 2, 2, 24, 6),
    (9, 1030, 16, 1, 32, 32), (70, 70, 3, 3, 16, 0), (77, 501, 3, 5, 64, 48), (50, 1, 7, 1, 8, 8),
    (1, 1, 1, 1, 8, 8), (1, 1, 8, 2, 64, 64), (3, 0, 4, 1, 32, 32), (0, 5, 4, 4, 40, 40),
    (7, 130, 3, 1, 40, 20),
    (257, 33, 16, 4, 128, 128), (65, 64, 2, 2, 80, 0), (31, 9, 5, 5, 96, 96), (10, 10, 4, 2, 24, 6), (5, 6, 2, 1, 8, 2),
    (4, 3, 1, 1, 104, 100), (12, 1, 33, 11, 16, 16), (6, 6, 8, 8, 128, 64), (9, 2, 4, 4, 120, 4), (2, 8, 1, 1, 112, 0),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nq,nk,hq,hk,d,rot", SHAPES)
def test_values_and_gradients(nq, nk, hq, hk, d, rot, dtype):
    q, k = heads(nq, hq, d, dtype, 1, 1.7), heads(nk, hk, d, dtype, 2, 0.3)
    g = torch.Generator().manual_seed(3)
    wq, wk = (1 + 0.3 * torch.randn(d, generator=g) for _ in range(2))
    pq, pk = (torch.randint(-50, 5000, (n,), generator=g, dtype=torch.int32).cuda() for n in (nq, nk))
    a, wq, wk = angles(rot), wq.cuda(), wk.cuda()
    kw = dict(q_weight=wq, k_weight=wk, q_positions=pq, k_positions=pk, angles=a, eps=1e-5)
    oq, ok = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    same.same_qk_norm(q, k, oq, ok, **kw)
    check("q", oq, *reference(q, wq, pq, a, 1e-5))
    check("k", ok, *reference(k, wk, pk, a, 1e-5))
    dyq, dyk = heads(nq, hq, d, dtype, 4), heads(nk, hk, d, dtype, 5)
    dq, dk = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    dwq, dwk = torch.full_like(wq, float("nan")), torch.full_like(wk, float("nan"))
    ws = torch.full((max(1, same.same_qk_norm_workspace_size(d, nq, hq, nk, hk)),), 255, dtype=torch.uint8, device="cuda")
    same.same_qk_norm_backward(q, k, dyq, dyk, dq, dk, dwq, dwk, ws, **kw)
    for name, x, w, p, dy, dx, dw in (("q", q, wq, pq, dyq, dq, dwq), ("k", k, wk, pk, dyk, dk, dwk)):
        (want, bound), (want_w, bound_w) = reference(x, w, p, a, 1e-5, dy)
        check("d" + name, dx, want, bound)
        check("dw" + name, dw, want_w, bound_w)
    # without the weights' gradients: the same, and no workspace
    dq2, dk2 = torch.empty_like(q), torch.empty_like(k)
    same.same_qk_norm_backward(q, k, dyq, dyk, dq2, dk2, None, None, None, **kw)
    assert torch.equal(dq, dq2) and torch.equal(dk, dk2)


@pytest.mark.parametrize("nq,nk,hq,hk,d,rot", [
    (350, 350, 32, 8, 128, 128), (1, 1, 64, 8, 128, 128), (1, 1, 2, 64, 64, 64), (5, 3, 5, 7, 128, 126),
    (2, 900, 24, 5, 104, 100), (3, 2, 65, 17, 40, 40)])
def test_few_tokens_of_unlike_heads(nq, nk, hq, hk, d, rot):
    """A token's heads go over several waves, as many as the side with more heads has: the other
    side's heads are fewer than its waves, and nothing behind them is read."""
    q, k = heads(nq, hq, d, torch.bfloat16, 1), heads(nk, hk, d, torch.bfloat16, 2)
    pq, pk = (torch.arange(n, dtype=torch.int32, device="cuda") for n in (nq, nk))
    oq, ok = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    same.same_qk_norm(q, k, oq, ok, q_positions=pq, k_positions=pk, angles=angles(rot))
    check("q", oq, *reference(q, None, pq, angles(rot), 1e-6))
    check("k", ok, *reference(k, None, pk, angles(rot), 1e-6))


@pytest.mark.parametrize("d,rot", [(72, 2), (128, 0)])
def test_sums_of_many_tokens(d, rot):
    """The weights' gradients of 2^24 equal tokens, whose roundings all go one way.  Sums are
    16 terms in 32 bits, then 64, with one rounding of a part and one of the result: 18 U of
    the terms beside the terms' own errors, whatever their number."""
    n = 1 << 24
    q, dy, k = heads(1, 1, d, torch.bfloat16, 1), heads(1, 1, d, torch.bfloat16, 2), heads(0, 1, d, torch.bfloat16, 3)
    pos, dw = torch.full((n,), 3, dtype=torch.int32, device="cuda"), torch.empty(d, device="cuda")
    dq = torch.empty(n, 1, d, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(same.same_qk_norm_workspace_size(d, n, 1, 0, 1), dtype=torch.uint8, device="cuda")
    same.same_qk_norm_backward(q.expand(n, 1, d), k, dy.expand(n, 1, d), k, dq, k, dw, None, ws, q_positions=pos,
                               k_positions=pos[:0], angles=angles(rot))
    _, (want, bound) = reference(q, None, pos[:1], angles(rot), 1e-6, dy)   # of one token: its terms' errors, and U
    check("dw", dw, n * want, n * (bound + 18 * U * want.abs()))


def test_no_tokens():
    q, k = heads(0, 2, 32, torch.float16, 1), heads(0, 1, 32, torch.float16, 2)
    w = torch.ones(32, device="cuda")
    same.same_qk_norm(q, k, q.clone(), k.clone(), q_weight=w)
    dw = torch.full((2, 32), float("nan"), device="cuda")
    same.same_qk_norm_backward(q, k, q, k, q.clone(), k.clone(), dw[0], dw[1], None, q_weight=w)
    assert not dw.any()


def test_gradient_against_differences():
    """fp32, one head: central differences of the loss sum(y dy)."""
    q = heads(3, 2, 24, torch.float32, 1).double().float()
    k, dy = heads(1, 1, 24, torch.float32, 2), heads(3, 2, 24, torch.float32, 3)
    w = (1 + 0.1 * torch.arange(24)).float().cuda()
    pos = torch.tensor([0, 7, 300], dtype=torch.int32, device="cuda")
    kw = dict(q_weight=w, q_positions=pos, k_positions=pos[:1], angles=angles(24), eps=1e-6)
    dq, dk, dw = torch.empty_like(q), torch.empty_like(k), torch.empty_like(w)
    ws = torch.empty(same.same_qk_norm_workspace_size(24, 3, 2, 1, 1), dtype=torch.uint8, device="cuda")
    same.same_qk_norm_backward(q, k, dy, k, dq, dk, dw, None, ws, **kw)

    def loss(q, w):
        y, _ = reference(q, w, pos, angles(24), 1e-6)
        return float((y * dy.cpu().double()).sum())

    h = 1e-5   # of 64-bit differences: h^2 and 2^-52 / h of the loss's size, below 1e-8
    for at in ((0, 0, 0), (1, 1, 13), (2, 0, 23)):
        e = torch.zeros(3, 2, 24, dtype=torch.float64)
        e[at] = h
        slope = (loss(q.cpu().double() + e, w) - loss(q.cpu().double() - e, w)) / (2 * h)
        assert abs(slope - float(dq[at])) < 1e-5 * max(1.0, abs(slope))
    for at in (0, 12, 23):
        e = torch.zeros(24, dtype=torch.float64)
        e[at] = h
        slope = (loss(q, w.cpu().double() + e) - loss(q, w.cpu().double() - e)) / (2 * h)
        assert abs(slope - float(dw[at])) < 1e-5 * max(1.0, abs(slope))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strides(dtype):
    """q, k as parts of one projection, transposed heads, repeated rows."""
    buf = heads(50, 12, 64, dtype, 1)
    q, k = buf[:, :8], buf[:, 8:]
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    kw = dict(q_positions=pos, k_positions=pos, angles=angles(64))
    want = [torch.empty(50, 8, 64, dtype=dtype, device="cuda"), torch.empty(50, 4, 64, dtype=dtype, device="cuda")]
    same.same_qk_norm(q.contiguous(), k.contiguous(), *want, **kw)
    got = [torch.empty_like(w) for w in want]
    same.same_qk_norm(q, k, *got, **kw)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    t = q.transpose(0, 1).contiguous().transpose(0, 1)
    same.same_qk_norm(t, k, *got, **kw)
    assert torch.equal(got[0], want[0])
    one = k[:1].expand(50, 4, 64)
    same.same_qk_norm(q, one, got[0], got[1], **kw)
    same.same_qk_norm(q, one.contiguous(), want[0], want[1], **kw)
    assert torch.equal(got[1], want[1])
    # the gradient's strided inputs
    dy = torch.cat([buf, buf], dim=2)[:, :8, 32:96]
    ws = torch.empty(same.same_qk_norm_workspace_size(64, 50, 8, 50, 4), dtype=torch.uint8, device="cuda")
    res = []
    for a, b, c in ((q, k, dy), (q.contiguous(), k.contiguous(), dy.contiguous())):
        dq, dk, dw = torch.empty_like(want[0]), torch.empty_like(want[1]), torch.empty(64, device="cuda")
        same.same_qk_norm_backward(a, b, c, b, dq, dk, dw, None, ws, **kw)
        res.append((dq, dk, dw))
    assert all(torch.equal(x, y) for x, y in zip(*res))


def test_in_place():
    q, k = heads(37, 4, 80, torch.float16, 1), heads(20, 2, 80, torch.float16, 2)
    pos = torch.arange(37, dtype=torch.int32, device="cuda")
    kw = dict(q_positions=pos, k_positions=pos[:20], angles=angles(80))
    want = torch.empty_like(q), torch.empty_like(k)
    same.same_qk_norm(q, k, *want, **kw)
    a, b = q.clone(), k.clone()
    same.same_qk_norm(a, b, a, b, **kw)
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])
    dq, dk = torch.empty_like(q), torch.empty_like(k)
    same.same_qk_norm_backward(q, k, a, b, dq, dk, None, None, None, **kw)
    same.same_qk_norm_backward(q, k, a, b, a, b, None, None, None, **kw)
    assert torch.equal(a, dq) and torch.equal(b, dk)


@pytest.mark.parametrize("far", [1 << 24, (1 << 31) - 1, -(1 << 31)])
def test_far_positions(far):
    """Angles of 2^31 radians and more keep their place in the turn: 64 bits
    round the reference's own angle to 2^-22, so integers of turns are used."""
    turns = np.array([0.5, 0.25, 0.125, 1.0]) * 2 * np.pi
    q = heads(1, 2, 8, torch.float32, 1)
    pos = torch.tensor([far], dtype=torch.int32, device="cuda")
    got, k = torch.empty_like(q), heads(0, 1, 8, torch.float32, 2)
    same.same_qk_norm(q, k, got, k, q_positions=pos, k_positions=pos[:0], angles=turns)
    # 2 pi in 64 bits is off by 2^-54 of itself: position 2^31 by 2^-22 radians, of which the exact place is known
    off = (2 * np.pi / (6.283185307179586476925286766559) - 1.0)
    assert abs(off) < 2.0 ** -52
    whole = torch.tensor([(far * n) % 8 / 8 for n in (4, 2, 1, 8)], dtype=torch.float64) * 2 * np.pi
    x = q.cpu().double()
    z = x / (x.square().mean(-1, keepdim=True) + float(np.float32(1e-6))).sqrt()
    want = torch.cat([z[..., :4] * whole.cos() - z[..., 4:] * whole.sin(),
                      z[..., 4:] * whole.cos() + z[..., :4] * whole.sin()], dim=-1)
    room = abs(far) * 2 * np.pi * 2.0 ** -53 + 32 * U
    assert bool(((got.cpu().double() - want).abs() <= room * (z[..., :4].abs() + z[..., 4:].abs()).repeat(1, 1, 2)).all())


@pytest.mark.parametrize("far", [1, 1000, -(1 << 20), (1 << 31) - 1])
def test_large_angles(far):
    """Angles of many turns a position: their place in the turn from 60 digits of pi."""
    two_pi = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459")
    turns = np.array([0.7, -3.5, 12345.678, 1e9 + 0.1, -1e12 - 0.3, 2.0 ** 40, 500.25, 1e6 + 0.7])
    q, k = heads(1, 2, 16, torch.float32, 1), heads(0, 1, 16, torch.float32, 2)
    pos, got = torch.tensor([far], dtype=torch.int32, device="cuda"), torch.empty_like(q)
    same.same_qk_norm(q, k, got, k, q_positions=pos, k_positions=pos[:0], angles=turns)
    place = torch.tensor([float(Fraction(a) * far / two_pi % 1) for a in turns], dtype=torch.float64) * 2 * np.pi
    x = q.cpu().double()
    z = x / (x.square().mean(-1, keepdim=True) + float(np.float32(1e-6))).sqrt()
    want = torch.cat([z[..., :8] * place.cos() - z[..., 8:] * place.sin(),
                      z[..., 8:] * place.cos() + z[..., :8] * place.sin()], dim=-1)
    room = 32 * U + abs(far) * 2 * np.pi * 2.0 ** -63   # a turn's 64 bits, of at most half of one, twice rounded
    assert bool(((got.cpu().double() - want).abs() <= room * (z[..., :8].abs() + z[..., 8:].abs()).repeat(1, 1, 2)).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_huge_tiny_and_missing_values(dtype):
    q = heads(6, 1, 64, dtype, 1).float()
    q[0] *= 1e30    # squares pass 32 bits
    q[1] *= 1e-30   # squares vanish: eps decides
    q[2] = 0
    q[3, 0, 5] = float("nan")
    q[4, 0, 5] = float("inf")
    q = q.to(dtype)
    k, pos = q[:0], torch.zeros(6, dtype=torch.int32, device="cuda")
    y, dx = torch.empty_like(q), torch.empty_like(q)
    kw = dict(q_positions=pos, k_positions=pos[:0], angles=angles(64))
    same.same_qk_norm(q, k, y, k, **kw)
    want, bound = reference(q, None, pos, angles(64), 1e-6)
    for row in (0, 1, 2, 5):
        check("row %d" % row, y[row], want[row], bound[row])
    assert bool(y[3].isnan().all()) and bool(y[4, 0, 5].isnan())
    dy = heads(6, 1, 64, dtype, 2)
    same.same_qk_norm_backward(q, k, dy, k, dx, k, None, None, None, **kw)
    (want, bound), _ = reference(q, None, pos, angles(64), 1e-6, dy)
    for row in (0, 1, 2, 5):
        check("row %d" % row, dx[row], want[row], bound[row])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,rot", [(128, 128), (64, 0), (40, 20), (8, 2)])
def test_the_largest_values(d, rot, dtype):
    """Heads up to the type's largest number in every element, and an eps that passes 32 bits
    together with the squares.  The gradient's own factor, 1 / |x|, is below the normal numbers
    there and held to 2^-22 of itself, within the bound's room of 24 U for 18."""
    big = torch.finfo(dtype).max
    q = heads(9, 2, d, dtype, 1).float()
    q[0] = torch.where(q[0] < 0, -big, big)
    q[1] = 0
    q[1, :, :2] = big
    q[2] = min(3.1e37, big)
    q[3] *= big / 8
    q[4] = min(1e19, big)
    q[5] *= min(1e19, big / 8)
    q[6] = 0
    q[6, :, 1] = -big
    q[7] *= min(3e18, big / 8)
    q = q.clamp(-big, big).to(dtype)
    w = (1 + 0.1 * torch.arange(d)).float().cuda()
    pos, a = torch.arange(9, dtype=torch.int32, device="cuda"), angles(rot)
    k, dy = q[:0], (1000 * heads(9, 2, d, dtype, 2).float()).clamp(-big, big).to(dtype)
    ws = torch.empty(same.same_qk_norm_workspace_size(d, 9, 2, 0, 2), dtype=torch.uint8, device="cuda")
    for eps in (1e-6, 3e38):
        kw = dict(q_weight=w, q_positions=pos, k_positions=pos[:0], angles=a, eps=eps)
        y, dx, dw = torch.empty_like(q), torch.empty_like(q), torch.empty_like(w)
        same.same_qk_norm(q, k, y, k, **kw)
        same.same_qk_norm_backward(q, k, dy, k, dx, k, dw, None, ws, **kw)
        check("y", y, *reference(q, w, pos, a, eps))
        (want, bound), (want_w, bound_w) = reference(q, w, pos, a, eps, dy)
        check("dx", dx, want, bound)
        check("dw", dw, want_w, bound_w)


def test_far_offsets():
    """More than 2^31 elements, and a view whose rows lie as far apart: a row's result is its own."""
    n = 2_100_000
    q = torch.zeros(n, 8, 128, dtype=torch.bfloat16, device="cuda")
    q.view(-1)[:1 << 20].normal_()
    q[-5:] = heads(5, 8, 128, torch.bfloat16, 3)
    dy, k = q, heads(0, 1, 128, torch.bfloat16, 1)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    kw = dict(k_positions=pos[:0], angles=angles(64))
    y = torch.empty_like(q)
    same.same_qk_norm(q, k, y, k.clone(), q_positions=pos, **kw)
    want = torch.empty_like(q[-5:])
    same.same_qk_norm(q[-5:], k, want, k.clone(), q_positions=pos[-5:], **kw)
    assert torch.equal(y[-5:], want)
    same.same_qk_norm_backward(q, k, dy, k, y, k.clone(), None, None, None, q_positions=pos, **kw)
    same.same_qk_norm_backward(q[-5:], k, dy[-5:], k, want, k.clone(), None, None, None, q_positions=pos[-5:], **kw)
    assert torch.equal(y[-5:], want)
    far = q.view(-1).as_strided((2, 2, 128), (n * 1024 - 2048, 1024, 1))   # the first and the last two tokens' first heads
    got = torch.empty(2, 2, 128, dtype=q.dtype, device="cuda")
    same.same_qk_norm(far, k, got, k.clone(), q_positions=pos[:2], **kw)
    again = torch.empty_like(got)
    same.same_qk_norm(far.contiguous(), k, again, k.clone(), q_positions=pos[:2], **kw)
    assert torch.equal(got, again) and bool(got[1].float().abs().sum() > 0)


def test_streams_graphs_and_repeats():
    q, k = heads(300, 8, 64, torch.bfloat16, 1), heads(200, 2, 64, torch.bfloat16, 2)
    pos = torch.arange(300, dtype=torch.int32, device="cuda")
    w = torch.rand(64, device="cuda")
    kw = dict(q_weight=w, k_weight=w, q_positions=pos, k_positions=pos[:200], angles=angles(64))
    out = [torch.empty_like(x) for x in (q, k, q, k)] + [torch.empty(64, device="cuda") for _ in range(2)]
    ws = torch.empty(same.same_qk_norm_workspace_size(64, 300, 8, 200, 2), dtype=torch.uint8, device="cuda")

    def both():
        same.same_qk_norm(q, k, out[0], out[1], **kw)
        same.same_qk_norm_backward(q, k, out[0], out[1], *out[2:], ws, **kw)

    both()
    want = [o.clone() for o in out]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
    for seed in (7, 8, 7):
        q.copy_(heads(300, 8, 64, torch.bfloat16, seed))
        for o in out:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in out]
        both()
        assert all(torch.equal(a, b) for a, b in zip(got, out))
    assert not torch.equal(got[0], want[0])


def test_refusals():
    q, k = heads(4, 2, 64, torch.float16, 1), heads(3, 1, 64, torch.float16, 2)
    pos = torch.arange(4, dtype=torch.int32, device="cuda")
    w = torch.ones(64, device="cuda")
    ok = dict(q=q, k=k, q_out=torch.zeros_like(q), k_out=torch.zeros_like(k), q_weight=w, q_positions=pos,
              k_positions=pos[:3], angles=angles(64))

    def refuse(code=same.SAME_EINVAL, **kw):
        with pytest.raises(same.SameError) as e:
            same.same_qk_norm(**dict(ok, **kw))
        assert e.value.code == code and str(e.value)

    refuse(q=q.cpu())
    refuse(q=q.double())
    refuse(q=q[:, 0])
    refuse(k=k.float())
    refuse(k=k[..., :32])
    refuse(q=q.transpose(1, 2).contiguous().transpose(1, 2))
    refuse(q_out=ok["q_out"][:3])
    refuse(q_out=torch.zeros(4, 2, 128, dtype=torch.float16, device="cuda")[..., :64])
    refuse(q_weight=w[:32])
    refuse(q_weight=w.half())
    refuse(q_positions=pos[:3])
    refuse(q_positions=pos.long())
    refuse(q_positions=None)
    refuse(angles=angles(66))
    refuse(angles=np.full(32, np.nan))
    refuse(angles=np.ones((4, 4)))
    refuse(eps=0.0)
    refuse(eps=float("nan"))
    refuse(k_out=ok["q_out"].view(-1)[:192].view(3, 1, 64))
    refuse(q_out=k.expand(3, 2, 64).contiguous()[:0])
    buf = torch.zeros(1024, dtype=torch.float16, device="cuda")
    refuse(q=buf[:512].view(4, 2, 64), q_out=buf[64:576].view(4, 2, 64))
    refuse(same.SAME_EALIGN, q=torch.zeros(513, dtype=torch.float16, device="cuda")[1:].view(4, 2, 64))
    refuse(same.SAME_EALIGN, q=torch.zeros(4, 2, 65, dtype=torch.float16, device="cuda")[..., :64])
    assert not ok["q_out"].any() and not ok["k_out"].any()
    ws = torch.empty(1, dtype=torch.uint8, device="cuda")
    with pytest.raises(same.SameError, match="workspace"):
        same.same_qk_norm_backward(q, k, q, k, torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(w), None, ws,
                                   q_weight=w, q_positions=pos, k_positions=pos[:3], angles=angles(64))
