"""Calls of more than 2^32 threads, which no single launch takes."""
import numpy as np
import pytest
import torch

import paper_1511_06416_amd as same
from tests import cross_reference as ref
from workloads import make_network

pytestmark = pytest.mark.gpu
HF = torch.float16


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


def rows_kept(first, cols, drop, seed, call_id):
    """Keep flags of a row that begins at element `first`."""
    e = np.arange(first, first + cols, dtype=np.uint64)
    g = np.unique(e // np.uint64(8))
    w = ref.philox(g & np.uint64(0xFFFFFFFF), g >> np.uint64(32), np.uint64(4 << 24), np.uint64(call_id), seed)
    half = np.stack([(w >> np.uint64(s)) & np.uint64(0xFFFF) for s in (0, 16)], axis=-1).reshape(-1)
    at = int(e[0] - g[0] * np.uint64(8))
    return torch.from_numpy(half[at:at + cols] >= round(drop * 65536))


@pytest.mark.parametrize("cols", [1 << 20, (1 << 20) - 1])
def test_dropout_of_more_than_2_to_35_elements(cols):
    """In place; groups of eight whose number passes 32 bits, in whole rows and
    in rows that are not."""
    rows = (1 << 15) + 3
    x = torch.ones(rows, 1 << 20, dtype=HF, device="cuda")[:, :cols]
    same.same_dropout(x, x, 0.25, 4, 9)
    torch.cuda.synchronize()
    for r in (0, 1, 4095, 4096, 8192, 16383, 16384, 24576, 32767, 32768, rows - 1):
        keep = rows_kept(r * cols, cols, 0.25, 4, 9)
        got = x[r].cpu()
        assert torch.equal(got > 0, keep), r
        assert torch.equal(got[keep], torch.full_like(got[keep], 1 / 0.75)), r


def test_attention_of_more_than_2_to_25_blocks():
    """One key a segment: out is its value, dv the query's gradient."""
    heads, segs = 8192, 4200
    ql, kl = np.ones(segs, np.int64), np.ones(segs, np.int64)
    kl[0] = 33   # not a plan of small segments
    q_ptr, k_ptr = (np.concatenate([[0], np.cumsum(x)]) for x in (ql, kl))
    g = torch.Generator(device="cuda").manual_seed(0)
    q, dout = (torch.randn(segs, heads, 8, generator=g, device="cuda", dtype=HF) for _ in range(2))
    k, v = (torch.randn(segs + 32, heads, 8, generator=g, device="cuda", dtype=HF) for _ in range(2))
    plan = same.same_cross_create(q_ptr, k_ptr, heads, heads, 8, HF)
    ws = plan.new_workspace(backward=True)
    out, lse = torch.full_like(q, float("nan")), torch.full((segs, heads), float("nan"), device="cuda")
    dq, dk, dv = (torch.full_like(x, float("nan")) for x in (q, k, v))
    same.same_cross_attention(plan, q, k, v, out, lse, ws)
    same.same_cross_attention_backward(plan, q, k, v, out, lse, dout, dq, dk, dv, ws)
    assert torch.equal(out[1:], v[33:])
    assert torch.allclose(lse[1:], (q[1:].float() * k[33:].float()).sum(dim=2) * 8 ** -0.5, atol=1e-4)
    assert torch.equal(dv[33:], dout[1:])
    # dS = P (dP - delta) of one key: nothing but rounding
    assert float(dq[1:].abs().max()) < 1e-3 and float(dk[33:].abs().max()) < 1e-3
    cols = slice(0, 2)   # the longer segment's first heads
    want = ref.attention(*(x[:n, cols].cpu() for x, n in ((q, 1), (k, 33), (v, 33))), [0, 1], [0, 33], 8 ** -0.5, None,
                         0.0, 0, 0, dout[:1, cols].cpu())
    for n, x, m in (("out", out, 1), ("lse", lse, 1), ("dq", dq, 1), ("dk", dk, 33), ("dv", dv, 33)):
        ref.check(n, x[:m, cols], *want[n])


def test_small_segments_of_more_than_2_to_26_waves():
    """32 queries on one key: every row is the key's value."""
    heads, segs = 8192, 8200
    plan = same.same_cross_create(np.arange(segs + 1) * 32, np.arange(segs + 1), heads, heads, 8, HF)
    assert plan.workspace_bytes(True) == 0   # small segments
    g = torch.Generator(device="cuda").manual_seed(0)
    q = torch.randn(1, heads, 8, generator=g, device="cuda", dtype=HF).expand(32 * segs, heads, 8)
    k, v = (torch.randn(segs, heads, 8, generator=g, device="cuda", dtype=HF) for _ in range(2))
    out = torch.full(q.shape, float("nan"), device="cuda", dtype=HF)
    same.same_cross_attention(plan, q, k, v, out, None, None)
    for s in range(0, segs, 100):
        n = min(100, segs - s)
        assert torch.equal(out[32 * s:32 * (s + n)].view(n, 32, heads, 8), v[s:s + n, None].expand(n, 32, heads, 8)), s


def test_a_launch_that_would_run_short_is_refused():
    """The sampler's launches: growing five nodes of 860 million columns, whose
    states begin off the wide accesses' boundaries, takes 16.8 million blocks of
    256 threads; fewer columns work."""
    pptr, pidx, card = make_network(1).csr()
    ctx = same.same_create_ex(pptr, pidx, card, 1.0, state_bits=4)
    for ld, fits in ((4_000_000, True), (860_000_000, False)):
        src, dst = (torch.full((ctx.n_nodes * ld + 1,), v, dtype=torch.int16, device="cuda")[1:].view(ctx.n_nodes, 1, ld)
                    for v in (1, 0))
        if fits:
            same.same_grow_replicas(ctx, src, 1, dst, 4, ld)
            assert bool((dst == 0x1111).all())
        else:
            with pytest.raises(same.SameError) as e:
                same.same_grow_replicas(ctx, src, 1, dst, 4, ld)
            assert e.value.code == same.SAME_ESIZE
            assert not bool(dst.any())
        del src, dst
    ctx.close()
