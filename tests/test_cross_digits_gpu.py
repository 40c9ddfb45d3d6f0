"""fp16: keys that hardly count, and rows of many keys, keep the digits of their
type.  Probabilities down to 2^-20 of a row's largest (2^-28 in the gradient of
the values) are rounded relatively; in the units of the softmax itself they
would lie among fp16's subnormals, below 2^-14.

Bounds: every probability's rounding to 11 bits (u), its fp32 error (2^-16: the
scores here stay below 16, the sums below 2^19 terms in chains of some 2^8), a
hundredth on the product of both, and the output's own rounding."""
import numpy as np
import pytest
import torch

import paper_1511_06416_amd as same
from tests import cross_reference as ref
from tests.test_cross_gpu import ptrs, run

pytestmark = pytest.mark.gpu
HF = torch.float16
U, TINY, EP = ref.U[HF], ref.TINY[HF], 2.0 ** -16


def uneven(rows, keys, d, seed):
    """Every query scores 0 on every key but the first, on which it scores
    log(2^24 / 40.5) or nearly: the others weigh 40.5 of fp16's smallest steps
    each, which rounds by up to 1.2 %.  The first key's values are zero."""
    g = torch.Generator().manual_seed(seed)
    q = torch.ones(rows, 1, d, dtype=HF)
    k = torch.zeros(keys, 1, d, dtype=HF)
    k[0] = np.log(2.0 ** 24 / 40.5) / d
    v = (1 + torch.rand(keys, 1, d, generator=g)).to(HF) * 512
    v[0] = 0
    return q, k, v


@pytest.mark.parametrize("d", [8, 32, 64, 96, 128])
@pytest.mark.parametrize("rows,keys,heads", [(1, 20, 2), (5, 32, 1), (1, 500, 700), (300, 500, 40), (2100, 300, 64)])
def test_forward(d, rows, keys, heads):
    q, k, v = uneven(rows, keys, d, d + rows)
    p = torch.softmax(q[:1, 0].double() @ k[:, 0].double().T, dim=1)
    want = p @ v[:, 0].double()
    bound = 1.01 * (p * (U + EP)) @ v[:, 0].double() + U * want + TINY
    many = [x.cuda().expand(-1, heads, -1) for x in (q, k, v)]
    got = run(*many, [0, rows], [0, keys], scale=1.0)
    ref.check("out", got["out"], want[:, None].expand(rows, heads, d), bound[:, None].expand(rows, heads, d))
    lse = torch.logsumexp(q[:1, 0].double() @ k[:, 0].double().T, dim=1)
    assert float((got["lse"].cpu().double() - lse).abs().max()) <= 16 * EP


@pytest.mark.parametrize("d", [8, 32, 64, 96, 128])
@pytest.mark.parametrize("rows,keys,heads", [(5, 20, 2), (31, 32, 1), (40, 500, 3), (2, 700, 40)])
def test_value_gradient_of_keys_that_hardly_count(d, rows, keys, heads):
    q, k, v = uneven(rows, keys, d, d + rows)
    dout = (512 + 256 * torch.rand(rows, 1, d, generator=torch.Generator().manual_seed(1))).to(HF)
    p = torch.softmax(q[:, 0].double() @ k[:, 0].double().T, dim=1)
    want = p.T @ dout[:, 0].double()
    bound = 1.01 * (p * (U + EP)).T @ dout[:, 0].double() + U * want + TINY
    many = [x.cuda().expand(-1, heads, -1) for x in (q, k, v, dout)]
    got = run(*many[:3], [0, rows], [0, keys], many[3], scale=1.0)
    ref.check("dv", got["dv"], want[:, None].expand(keys, heads, d), bound[:, None].expand(keys, heads, d))


@pytest.mark.parametrize("d,drop", [(8, 0.0), (64, 0.0), (128, 0.0), (64, 0.25), (128, 0.25)])
@pytest.mark.parametrize("rows,keys", [(3, 166_938), (40, 166_938), (40, 414_252)])
def test_value_gradient_of_many_keys(d, drop, rows, keys):
    """Nearly equal weights of 100.5 and 40.5 of fp16's smallest steps."""
    if drop and keys > 200_000:
        pytest.skip("the definition's random numbers would take minutes")
    g = torch.Generator().manual_seed(d + rows)
    q = (torch.randn(rows, 1, d, generator=g) * 1e-3).to(HF)
    k, v = (torch.randn(keys, 1, d, generator=g).to(HF) for _ in range(2))
    dout = (512 + 256 * torch.rand(rows, 1, d, generator=g)).to(HF)
    p = torch.softmax(q[:, 0].double() @ k[:, 0].double().T * d ** -0.5, dim=1)
    if drop:
        p = p * ref.attention_keep(np.arange(rows), 0, 1, keys, drop, 11, 3)
    want = p.T @ dout[:, 0].double()
    bound = 1.01 * (p * (U + EP)).T @ dout[:, 0].double() + U * want + TINY
    dev = [x.cuda() for x in (q, k, v, dout)]
    got = run(*dev[:3], [0, rows], [0, keys], dev[3], drop=drop)
    ref.check("dv", got["dv"], want[:, None], bound[:, None])
    assert all(bool(x.isfinite().all()) for x in got.values())


@pytest.mark.parametrize("keys", [2, 40, 300])
def test_certain_keys_stay_in_range(keys):
    """A probability of one, and score gradients of half of fp16's range."""
    q, k = torch.ones(3, 1, 64, dtype=HF), torch.zeros(keys, 1, 64, dtype=HF)
    k[0] = 1
    v = torch.zeros_like(k)
    v[0], v[1] = 60, -60
    dout = torch.full_like(q, 8)
    dev = [x.cuda() for x in (q, k, v, dout)]
    for scale in (4.0, 2.0 ** -10):   # one key takes all; all alike
        want = ref.attention(q, k, v, [0, 3], [0, keys], scale, None, 0.0, 11, 3, dout)
        got = run(*dev[:3], ptrs([3]), ptrs([keys]), dev[3], scale=scale)
        for n in got:
            assert bool(got[n].isfinite().all()), n
            ref.check(n, got[n], *want[n])


@pytest.mark.parametrize("d", [8, 64, 128])
@pytest.mark.parametrize("rows,keys,heads", [(5, 20, 2), (1, 500, 3), (300, 500, 40), (2100, 300, 64)])
@pytest.mark.parametrize("size", [300.0, 5000.0, 3e4])
@pytest.mark.parametrize("dtype", [HF, torch.bfloat16])
def test_forward_of_huge_scores(d, rows, keys, heads, size, dtype):
    """Scores of 2^17 to 2^34, where fp32 has no digits below 1 left: the key
    on which they are largest takes all, and out is its value exactly."""
    q = torch.full((rows, 1, d), size).to(dtype)
    k = torch.full((keys, 1, d), 0.75 * size).to(dtype)
    v = torch.randn(keys, 1, d, generator=torch.Generator().manual_seed(d)).to(dtype)
    for best in (0, keys // 2, keys - 1):
        kk = k.clone()
        kk[best] = size
        got = run(*(x.cuda().expand(-1, heads, -1) for x in (q, kk, v)), [0, rows], [0, keys])
        assert torch.equal(got["out"].cpu(), v[best].expand(rows, heads, d)), best
        lse = float((q[0, 0].double() * kk[best, 0].double()).sum()) * d ** -0.5
        assert float((got["lse"].double() - lse).abs().max()) <= 2.0 ** -21 * lse, best
