"""Cross attention and dropout, as measured cases.

The operators of an amortised imputer beside the sampler: a column's missing
entries (queries) attend to the same column's known entries (keys and values,
of another length), and training drops attention probabilities and branch
values with the counter-based generator.  A case is one pass: the attention of
a prediction (`attend`), the attention with its gradients (`train`), dropout
with the residual sum (`dropout`) or dropout with its gradient
(`dropout_train`).  Numbers of nodes, hidden shares and columns are those of
the repository's workloads; heads, widths and long lengths are generic.

`own` chooses between the plain forms (elementary torch operations in 32
bits) and the package's operators.  `exact` repeats a pass from the definition
in 64 bits and uses nothing of the package.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
MAX_FLOPS = 5.4e11     # the longest listed attention
MAX_BYTES = 1.3e9      # the longest listed cache
CALL_ID = 7


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # one missing answer of one 330-node column, asked for alone: latency
        dict(name="attend one entry", do="attend", form="long", segs=1, q=1, k=301, ragged=False, hq=8, hkv=2, d=64,
             dtype="bf16", hidden=0.0, drop=0.0),
        # a minibatch of the five-node student network, half hidden: many tiny
        # columns, some with nothing known and some with nothing missing
        dict(name="attend student 2k", do="attend", form="nodes", segs=2_000, nodes=5, missing=0.5, hq=4, hkv=4, d=32,
             dtype="fp16", hidden=0.0, drop=0.0, len_seed=1),
        # two-layer assessment network, known entries held out at random
        dict(name="attend concepts 256", do="attend", form="nodes", segs=256, nodes=330, missing=0.5, hq=8, hkv=8,
             d=64, dtype="fp16", hidden=0.1, drop=0.0, len_seed=2),
        # thousand-node network, the forward pass of training, shared key heads
        dict(name="attend thousand 64 drop", do="attend", form="nodes", segs=64, nodes=1000, missing=0.4, hq=16,
             hkv=4, d=64, dtype="bf16", hidden=0.0, drop=0.1, len_seed=3),
        # single queries over long contexts (many columns as one context):
        # every key and value is read once, for four query heads
        dict(name="attend single long", do="attend", form="long", segs=16, q=1, k=20_011, ragged=True, hq=32, hkv=8,
             d=128, dtype="bf16", hidden=0.0, drop=0.0, len_seed=4),
        # the largest: thousands of queries over a long context
        dict(name="attend long", do="attend", form="long", segs=2, q=4_099, k=7_951, ragged=False, hq=16, hkv=4,
             d=128, dtype="bf16", hidden=0.0, drop=0.0),
        # training steps: forward with dropout, then every gradient
        dict(name="train student 2k", do="train", form="nodes", segs=2_000, nodes=5, missing=0.5, hq=4, hkv=4, d=32,
             dtype="fp16", hidden=0.0, drop=0.1, len_seed=5),
        dict(name="train concepts 128", do="train", form="nodes", segs=128, nodes=330, missing=0.5, hq=8, hkv=8,
             d=64, dtype="bf16", hidden=0.1, drop=0.1, len_seed=6),
        dict(name="train long", do="train", form="long", segs=1, q=4_099, k=4_095, ragged=False, hq=16, hkv=4,
             d=128, dtype="bf16", hidden=0.0, drop=0.0),
        # dropout on the residual branch: a few columns, a large minibatch, and
        # rows inside a wider buffer with the gradient
        dict(name="dropout small", do="dropout", rows=257, cols=330, row_stride=330, residual=True, dtype="bf16",
             drop=0.1),
        dict(name="dropout large", do="dropout", rows=65_536, cols=1_024, row_stride=1_024, residual=True,
             dtype="bf16", drop=0.1),
        dict(name="dropout rows train", do="dropout_train", rows=20_003, cols=1_000, row_stride=1_024,
             residual=False, dtype="fp32", drop=0.25),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, costing no more than the listed."""
    kind = rng.choice(["attend", "attend", "train", "dropout", "dropout_train"])
    if kind.startswith("dropout"):
        dtype = rng.choice(["bf16", "fp16", "fp32"])
        rows, cols = _log(rng, 1, 60_000), _log(rng, 5, 1_030)
        stride = cols + rng.choice([0, 0, 1, 8, 24])
        return dict(do=kind, rows=rows, cols=cols, row_stride=stride, residual=rng.random() < 0.5, dtype=dtype,
                    drop=rng.choice([0.1, 0.25, 0.5]))
    hkv = rng.choice([1, 2, 4, 8])
    base = dict(do=kind, hq=hkv * rng.choice([1, 1, 2, 4]), hkv=hkv, d=rng.choice([32, 40, 64, 64, 80, 96, 128, 128]),
                dtype=rng.choice(["bf16", "fp16"]), hidden=rng.choice([0.0, 0.0, 0.1, 0.5]),
                drop=rng.choice([0.0, 0.1, 0.25]), len_seed=rng.randrange(1 << 30))
    while True:
        case = dict(base)
        form = rng.choice(["nodes", "long", "single"])
        if form == "nodes":
            nodes = rng.choice([5, 100, 330, 1000])
            case.update(form="nodes", segs=_log(rng, 1, 200_000 // (4 * nodes)), nodes=nodes,
                        missing=rng.choice([0.3, 0.4, 0.5, 0.9]))
        elif form == "long":
            case.update(form="long", segs=rng.randint(1, 4), q=_log(rng, 2, 4_100), k=_log(rng, 2, 8_000),
                        ragged=rng.random() < 0.7)
        else:
            case.update(form="long", segs=_log(rng, 1, 32), q=1, k=_log(rng, 1, 32_000), ragged=rng.random() < 0.7)
        ql, kl = _lengths(case)
        scores = int((ql * kl).sum()) * case["hq"]
        w = work(case)
        if (sum(ql) and sum(kl) and w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES and scores <= 5.4e8
                and case["segs"] * int(ql.max()) * int(kl.max()) * case["hq"] <= 1.2e9):
            return case


def _lengths(case):
    """Queries and keys of every segment; the column structure is fixed, like a
    data set's pattern of known entries, whatever the seed."""
    if case["form"] == "nodes":
        r = np.random.default_rng(case["len_seed"])
        ql = r.binomial(case["nodes"], case["missing"], size=case["segs"]).astype(np.int64)
        return ql, case["nodes"] - ql
    ql = np.full(case["segs"], case["q"], np.int64)
    kl = np.full(case["segs"], case["k"], np.int64)
    if case["ragged"]:
        r = np.random.default_rng(case["len_seed"])
        kl = np.maximum(1, (kl * r.uniform(0.25, 1.0, size=case["segs"])).astype(np.int64))
        if case["q"] > 1:
            ql = np.maximum(1, (ql * r.uniform(0.25, 1.0, size=case["segs"])).astype(np.int64))
    return ql, kl


def work(case):
    if case["do"].startswith("dropout"):
        n = case["rows"] * case["cols"]
        size = 4 if case["dtype"] == "fp32" else 2
        passes = 4 if case["do"] == "dropout_train" else 2
        return {"bytes": n * size * (passes + (1 if case["residual"] else 0)), "flops": 2 * n}
    ql, kl = _lengths(case)
    tq, tk, d = int(ql.sum()), int(kl.sum()), case["d"]
    seen = float((ql * kl).sum()) * (1.0 - case["hidden"])
    rows, keys = tq * case["hq"] * d * 2, tk * case["hkv"] * d * 2
    mask = tk if case["hidden"] else 0
    if case["do"] == "attend":
        return {"bytes": 2 * rows + 2 * keys + mask, "flops": 4 * seen * case["hq"] * d}
    # q, k, v, dout read, out, dq, dk, dv written
    return {"bytes": 4 * rows + 4 * keys + mask, "flops": 14 * seen * case["hq"] * d}


# ----------------------------------------------------------------- the inputs

def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed((seed * 1_000_003 + 17) % (1 << 62))
    dt = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)

    rng_seed = (seed * 0x9E3779B97F4A7C15 + 0x1234567) & ((1 << 64) - 1)
    if case["do"].startswith("dropout"):
        n, c, s = case["rows"], case["cols"], case["row_stride"]
        x = normal(n, s)[:, :c]
        res = normal(n, s)[:, :c] if case["residual"] else None
        dy = normal(n, s)[:, :c] if case["do"] == "dropout_train" else None
        return dict(x=x, res=res, dy=dy, rng_seed=rng_seed)
    ql, kl = _lengths(case)
    tq, tk = int(ql.sum()), int(kl.sum())
    q, k, v = (normal(tq, case["hq"], case["d"]), normal(tk, case["hkv"], case["d"]),
               normal(tk, case["hkv"], case["d"]))
    mask = None
    if case["hidden"]:
        mask = (torch.rand(tk, generator=g, device="cuda") >= case["hidden"]).to(torch.uint8)
    dout = normal(tq, case["hq"], case["d"]) if case["do"] == "train" else None
    return dict(q=q, k=k, v=v, mask=mask, dout=dout, rng_seed=rng_seed, ql=ql, kl=kl,
                scale=1.0 / math.sqrt(case["d"]))


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if case["do"].startswith("dropout"):
        if own:
            st["y"] = torch.empty_strided(st["x"].shape, st["x"].stride(), dtype=st["x"].dtype, device="cuda")
            if st["dy"] is not None:
                st["dx"] = torch.empty_like(st["y"])
        return st
    q_ptr = np.concatenate([[0], np.cumsum(st["ql"])]).astype(np.int64)
    k_ptr = np.concatenate([[0], np.cumsum(st["kl"])]).astype(np.int64)
    if own:
        import paper_1511_06416_amd as same
        train = case["do"] == "train"
        st["plan"] = same.same_cross_create(q_ptr, k_ptr, case["hq"], case["hkv"], case["d"], st["q"].dtype)
        st["ws"] = st["plan"].new_workspace(backward=train)
        st["out"] = torch.empty_like(st["q"])
        if train:
            st["lse"] = torch.empty(st["q"].shape[:2], dtype=torch.float32, device="cuda")
            st["dq"], st["dk"], st["dv"] = (torch.empty_like(st[n]) for n in ("q", "k", "v"))
        return st
    # the plain form's plan: padded positions of every segment
    ql, kl = torch.from_numpy(st["ql"]).cuda(), torch.from_numpy(st["kl"]).cuda()
    qp, kp = torch.from_numpy(q_ptr[:-1]).cuda(), torch.from_numpy(k_ptr[:-1]).cuda()
    iq = torch.arange(int(st["ql"].max()), device="cuda")
    ik = torch.arange(int(st["kl"].max()), device="cuda")
    st["q_in"], st["k_in"] = iq[None] < ql[:, None], ik[None] < kl[:, None]
    st["q_at"] = torch.where(st["q_in"], qp[:, None] + iq[None], 0)
    st["k_at"] = torch.where(st["k_in"], kp[:, None] + ik[None], 0)
    return st


# ------------------------------------------------------------ the plain forms

def _philox(c0, c1, c2, c3, seed):
    """Philox4x32-10 on int64 tensors of 32-bit words; four such tensors."""
    low = 0xFFFFFFFF
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low)
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _keep_elements(shape, drop, seed):
    """Dropout's factors: element e of the matrix takes 16 bits, number e % 8
    of the block at counter {e / 8, high word, 4 << 24, call}."""
    n = shape[0] * shape[1]
    grp = torch.arange((n + 7) // 8, device="cuda")
    w = _philox(grp & 0xFFFFFFFF, grp >> 32, torch.full_like(grp, 4 << 24), torch.full_like(grp, CALL_ID), seed)
    half = torch.stack([(x >> s) & 0xFFFF for x in w for s in (0, 16)], dim=-1).reshape(-1)[:n].reshape(shape)
    t = int(round(drop * 65536))
    return (half >= t).to(torch.float32) * (65536.0 / (65536 - t))


def _keep_scores(rows, keys, drop, seed):
    """The attention's factors: key j of query row r (token * heads + head)
    takes 8 bits, byte j % 4 of word (j / 8) % 4 of the block at counter
    {2 (j / 32) + (j / 4) % 2, r, 3 << 24 | high word of r, call}."""
    n = (keys + 31) // 32
    c0 = torch.arange(2 * n, device="cuda").expand(rows.shape + (2 * n,))
    r = rows[..., None].expand(c0.shape)
    w = _philox(c0, r & 0xFFFFFFFF, (3 << 24) | (r >> 32), torch.full_like(c0, CALL_ID), seed)
    byte = torch.stack([torch.stack([(x >> s) & 0xFF for s in (0, 8, 16, 24)], dim=-1) for x in w], dim=-2)
    # [..., 32-key block, half, word, byte] -> key = block * 32 + word * 8 + half * 4 + byte
    byte = byte.reshape(rows.shape + (n, 2, 4, 4)).transpose(-3, -2).reshape(rows.shape + (32 * n,))[..., :keys]
    t = int(round(drop * 256))
    return (byte >= t).to(torch.float32) * (256.0 / (256 - t))


def _plain_dropout(st):
    case = st["case"]
    f = _keep_elements(st["x"].shape, case["drop"], st["rng_seed"])
    y = st["x"].float() * f
    if st["res"] is not None:
        y = y + st["res"].float()
    y = y.to(st["x"].dtype)
    if st["dy"] is None:
        return y
    f = _keep_elements(st["x"].shape, case["drop"], st["rng_seed"])
    return y, (st["dy"].float() * f).to(st["x"].dtype)


def _plain_attention(st):
    case = st["case"]
    b, lq = st["q_at"].shape
    lk = st["k_at"].shape[1]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    grp = hq // hkv
    dt = st["q"].dtype

    def by_query(x):   # [tokens, hq, d] -> [b, hkv, grp * lq, d]
        return x[st["q_at"]].float().reshape(b, lq, hkv, grp, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, grp * lq, d)

    def by_key(x):     # [tokens, hkv, d] -> [b, hkv, lk, d]
        return x[st["k_at"]].float().permute(0, 2, 1, 3).contiguous()

    def from_query(x):
        return x.reshape(b, hkv, grp, lq, d).permute(0, 3, 1, 2, 4).reshape(b, lq, hq, d)[st["q_in"]].to(dt)

    def from_key(x):
        return x.permute(0, 2, 1, 3)[st["k_in"]].to(dt)

    def factors():
        head = torch.arange(hq, device="cuda").reshape(1, hkv, grp, 1)
        rows = (st["q_at"].reshape(b, 1, 1, lq) * hq + head).reshape(b, hkv, grp * lq)
        return _keep_scores(rows, lk, case["drop"], st["rng_seed"])

    seen = st["k_in"] if st["mask"] is None else st["k_in"] & (st["mask"][st["k_at"]] != 0)
    q, k, v = by_query(st["q"]), by_key(st["k"]), by_key(st["v"])
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * st["scale"]
    s = s.masked_fill(~seen[:, None, None, :], float("-inf"))
    top = s.amax(dim=-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    del s
    total = p.sum(dim=-1, keepdim=True)
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    f = factors() if case["drop"] else None
    o = torch.matmul(p if f is None else p * f, v)
    out = from_query(o)
    if case["do"] == "attend":
        return out
    do = by_query(st["dout"])
    do = do * st["q_in"][:, None, None, :, None].expand(b, 1, grp, lq, 1).reshape(b, 1, grp * lq, 1)
    delta = (do * o).sum(dim=-1, keepdim=True)
    if case["drop"]:
        f = factors()
    dv = torch.matmul((p if f is None else p * f).transpose(2, 3).contiguous(), do)
    dp = torch.matmul(do, v.transpose(2, 3).contiguous())
    if f is not None:
        dp = dp * f
    ds = p * (dp - delta) * st["scale"]
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    return out, from_query(dq), from_key(dk), from_key(dv)


# ------------------------------------------------------------------- one pass

def run(state):
    case = state["case"]
    if not own:
        return _plain_dropout(state) if case["do"].startswith("dropout") else _plain_attention(state)
    import paper_1511_06416_amd as same
    if case["do"].startswith("dropout"):
        same.same_dropout(state["x"], state["y"], case["drop"], state["rng_seed"], CALL_ID, residual=state["res"])
        if state["dy"] is None:
            return state["y"]
        same.same_dropout(state["dy"], state["dx"], case["drop"], state["rng_seed"], CALL_ID)
        return state["y"], state["dx"]
    same.same_cross_attention(state["plan"], state["q"], state["k"], state["v"], state["out"], state.get("lse"),
                              state["ws"], key_mask=state["mask"], scale=state["scale"], drop=case["drop"],
                              seed=state["rng_seed"], call_id=CALL_ID)
    if case["do"] == "attend":
        return state["out"]
    same.same_cross_attention_backward(state["plan"], state["q"], state["k"], state["v"], state["out"], state["lse"],
                                       state["dout"], state["dq"], state["dk"], state["dv"], state["ws"],
                                       key_mask=state["mask"], scale=state["scale"], drop=case["drop"],
                                       seed=state["rng_seed"], call_id=CALL_ID)
    return state["out"], state["dq"], state["dk"], state["dv"]


# ---------------------------------------------------------- the 64-bit answer

def _philox_words(c0, c1, c2, c3, seed):
    """Philox4x32-10 over numpy arrays, from its published definition."""
    c0, c1, c2, c3 = np.broadcast_arrays(*(np.asarray(c, np.uint64) for c in (c0, c1, c2, c3)))
    low, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    key = [seed % (1 << 32), seed // (1 << 32)]
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c0, np.uint64(0xCD9E8D57) * c2
        c0 = (p1 >> sh) ^ c1 ^ np.uint64(key[0])
        c2 = (p0 >> sh) ^ c3 ^ np.uint64(key[1])
        c1, c3 = p1 & low, p0 & low
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    return np.stack([c0, c1, c2, c3], axis=-1).astype(np.uint32)


def _exact_dropout(case, st):
    n = case["rows"] * case["cols"]
    blocks = np.arange(-(-n // 8), dtype=np.uint64)
    words = _philox_words(blocks % (1 << 32), blocks // (1 << 32), 4 << 24, CALL_ID, st["rng_seed"])
    halves = np.ascontiguousarray(words).view(np.uint16).reshape(-1)[:n]   # little endian: the low half first
    dropped = int(round(case["drop"] * 65536))
    keep = torch.from_numpy((halves >= dropped).reshape(case["rows"], case["cols"])).cuda()
    gain = 65536.0 / (65536.0 - dropped)
    y = torch.where(keep, st["x"].double() * gain, 0.0)
    if st["res"] is not None:
        y = y + st["res"].double()
    return y if st["dy"] is None else (y, torch.where(keep, st["dy"].double() * gain, 0.0))


def exact(case, seed):
    st = _inputs(case, seed)
    if case["do"].startswith("dropout"):
        return _exact_dropout(case, st)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["drop"] and float((st["ql"] * st["kl"]).sum()) * hq > 4e8:
        return None
    train = case["do"] == "train"
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    grads = [torch.zeros(st[n].shape, dtype=torch.float64, device="cuda") for n in ("q", "k", "v")] if train else []
    dropped = int(round(case["drop"] * 256))
    q0 = k0 = 0
    for nq, nk in zip(st["ql"].tolist(), st["kl"].tolist()):
        qs, ks = slice(q0, q0 + nq), slice(k0, k0 + nk)
        visible = torch.arange(nk, device="cuda")
        if st["mask"] is not None:
            visible = visible[st["mask"][ks].bool()]
        if nq and len(visible):
            factor = None
            if dropped:
                j = np.arange(nk)
                rows = (np.arange(q0, q0 + nq)[:, None] * hq + np.arange(hq)[None]).astype(np.uint64)
                blocks = np.arange(-(-nk // 32) * 2, dtype=np.uint64)
                words = _philox_words(blocks, rows[..., None] % (1 << 32), (3 << 24) + rows[..., None] // (1 << 32),
                                      CALL_ID, st["rng_seed"])
                one = np.ascontiguousarray(words).view(np.uint8).reshape(nq, hq, len(blocks), 16)
                one = one[:, :, (j // 32) * 2 + (j // 4) % 2, ((j // 8) % 4) * 4 + j % 4]
                factor = torch.from_numpy(one >= dropped).cuda()[:, :, visible].double() * (256.0 / (256.0 - dropped))
            for g in range(hkv):
                kk, vv = st["k"][ks, g].double()[visible], st["v"][ks, g].double()[visible]
                for h in range(g * hq // hkv, (g + 1) * hq // hkv):
                    qq = st["q"][qs, h].double()
                    p = torch.softmax((qq @ kk.T) * st["scale"], dim=1)
                    fp = p if factor is None else p * factor[:, h]
                    o = fp @ vv
                    out[qs, h] = o
                    if train:
                        do = st["dout"][qs, h].double()
                        dp = do @ vv.T
                        if factor is not None:
                            dp = dp * factor[:, h]
                        ds = p * (dp - (p * dp).sum(dim=1, keepdim=True)) * st["scale"]
                        grads[0][qs, h] = ds @ kk
                        grads[1][ks, g] = grads[1][ks, g].index_add(0, visible, ds.T @ qq)
                        grads[2][ks, g] = grads[2][ks, g].index_add(0, visible, fp.T @ do)
        q0, k0 = q0 + nq, k0 + nk
    return tuple([out] + grads) if train else out
