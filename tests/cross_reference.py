"""Cross attention and dropout from their definitions, in 64 bits on the CPU,
with the bounds that rounding puts on the kernels' outputs."""
import numpy as np
import torch

# unit roundoffs: 8, 11 and 24 significant bits
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}   # half the smallest subnormal
F32 = 2.0 ** -18   # sums of up to 2^13 terms, exponents up to 2^6, in fp32: generous


def philox(c0, c1, c2, c3, seed):
    c0, c1, c2, c3 = (np.array(c, np.uint64) for c in np.broadcast_arrays(c0, c1, c2, c3))
    low, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c0, np.uint64(0xCD9E8D57) * c2
        c0, c1, c2, c3 = (b >> sh) ^ c1 ^ np.uint64(k0), b & low, (a >> sh) ^ c3 ^ np.uint64(k1), a & low
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack([c0, c1, c2, c3], axis=-1)


def attention_keep(tokens, head, heads, n_keys, drop, seed, call_id):
    """Factors of the query tokens (global numbers) of one head."""
    t = int(round(drop * 256))
    j = np.arange(n_keys)
    r = (np.asarray(tokens, np.uint64) * np.uint64(heads) + np.uint64(head))[:, None]
    w = philox((2 * (j // 32) + j // 4 % 2)[None].astype(np.uint64), r & np.uint64(0xFFFFFFFF),
               np.uint64(3 << 24) | (r >> np.uint64(32)), np.uint64(call_id), seed)
    word = np.take_along_axis(w, np.broadcast_to((j // 8 % 4)[None, :, None], w.shape[:2] + (1,)), axis=2)[..., 0]
    byte = (word >> (8 * (j % 4)).astype(np.uint64)[None]) & np.uint64(255)
    return torch.from_numpy((byte >= t).astype(np.float64) * (256.0 / (256 - t)))


def dropout_keep(rows, cols, drop, seed, call_id):
    t = int(round(drop * 65536))
    e = np.arange(rows * cols, dtype=np.uint64)
    g = e // np.uint64(8)
    w = philox(g & np.uint64(0xFFFFFFFF), g >> np.uint64(32), np.uint64(4 << 24), np.uint64(call_id), seed)
    word = np.take_along_axis(w, (e // np.uint64(2) % np.uint64(4)).astype(np.int64)[:, None], axis=1)[:, 0]
    half = (word >> (np.uint64(16) * (e % np.uint64(2)))) & np.uint64(0xFFFF)
    return torch.from_numpy(((half >= t) * (65536.0 / (65536 - t))).reshape(rows, cols))


def attention(q, k, v, q_ptr, k_ptr, scale, mask=None, drop=0.0, seed=0, call_id=0, dout=None):
    """Outputs in 64 bits and bounds on the kernels' errors: dict name ->
    (value, bound) for out, lse and, with dout, dq, dk, dv."""
    dt = q.dtype
    u, tiny = U[dt], TINY[dt]
    q, k, v = (x.detach().cpu().double() for x in (q, k, v))
    hq, hkv = q.shape[1], k.shape[1]
    res = {"out": torch.zeros_like(q), "lse": torch.full(q.shape[:2], -np.inf, dtype=torch.float64)}
    tol = {"out": torch.zeros_like(q), "lse": torch.zeros(q.shape[:2], dtype=torch.float64)}
    if dout is not None:
        dout = dout.detach().cpu().double()
        for n, x in (("dq", q), ("dk", k), ("dv", v)):
            res[n], tol[n] = torch.zeros_like(x), torch.zeros_like(x)
    mask = None if mask is None else mask.cpu().bool()
    for s in range(len(q_ptr) - 1):
        qs, ks = slice(q_ptr[s], q_ptr[s + 1]), np.arange(k_ptr[s], k_ptr[s + 1])
        local = np.arange(len(ks))
        if mask is not None:
            local = local[mask[ks].numpy()]
        ks = k_ptr[s] + local
        n_q = q_ptr[s + 1] - q_ptr[s]
        if n_q == 0 or len(ks) == 0:
            continue
        for h in range(hq):
            g = h // (hq // hkv)
            qq, kk, vv = q[qs, h], k[ks, g], v[ks, g]
            score = (qq @ kk.T) * scale
            p = torch.softmax(score, dim=1)
            f = torch.ones_like(p)
            if drop:
                f = attention_keep(np.arange(q_ptr[s], q_ptr[s + 1]), h, hq, k_ptr[s + 1] - k_ptr[s], drop, seed,
                                   call_id)[:, local]
            # relative error of a probability: fp32 scores, exponential and sum
            ep = F32 * (1 + (qq.abs() @ kk.abs().T * scale).amax(dim=1, keepdim=True))
            o = (p * f) @ vv
            res["out"][qs, h] = o
            # the rounding is to the unnormalised probability exp(s - max), whose tiny ones are
            # rounded absolutely; the sum is at least 1
            eo = (p * f * (u + ep)) @ vv.abs() + tiny * (f @ vv.abs())
            tol["out"][qs, h] = 1.01 * eo + u * o.abs() + tiny
            res["lse"][qs, h] = torch.logsumexp(score, dim=1)
            tol["lse"][qs, h] = (2 * ep[:, 0] + 2.0 ** -22 * res["lse"][qs, h].abs())
            if dout is None:
                continue
            do = dout[qs, h]
            dp = (do @ vv.T) * f
            delta = (do * o).sum(dim=1, keepdim=True)
            ds = p * (dp - delta)
            # delta is formed from the rounded out
            ed = ((tol["out"][qs, h]) * do.abs()).sum(dim=1, keepdim=True)
            mag = p * ((do.abs() @ vv.abs().T) * f + delta.abs())
            es = 1.01 * (u * ds.abs() + p * ed + (ep + F32) * mag) + tiny
            ev = (p * f * (u + ep) + tiny * f).T @ do.abs()
            res["dq"][qs, h] = (ds @ kk) * scale
            tol["dq"][qs, h] = es @ kk.abs() * scale * 1.01 + u * res["dq"][qs, h].abs() + tiny
            res["dk"][ks, g] += (ds.T @ qq) * scale
            tol["dk"][ks, g] += es.T @ qq.abs() * scale * 1.01
            res["dv"][ks, g] += (p * f).T @ do
            tol["dv"][ks, g] += 1.01 * ev
    if dout is not None:
        for n in ("dk", "dv"):
            tol[n] += u * res[n].abs() + tiny
    return {n: (res[n], tol[n]) for n in res}


def check(name, got, value, bound):
    """got within bound of value everywhere; infinities must be equal."""
    got = got.detach().cpu().double()
    inf = torch.isinf(value)
    assert torch.equal(got[inf], value[inf]), name
    off = (got - value).abs()[~inf]
    bad = ~(off <= bound[~inf])
    assert not bool(bad.any()), "%s: %d of %d out of bounds, worst %g over %g" % (
        name, int(bad.sum()), bad.numel(), float(off[bad].max()), float(bound[~inf][bad].min()))
