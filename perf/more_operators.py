"""The imputer's norms, answers and updates, as measured cases.

What a training step of the amortised imputer needs around its attention:
the norm of every query and key head with the rotation by position (`norm`),
the log probabilities of given states with entropy and the most likely
alternatives (`answers`), and the orthogonalised update of its matrices by
Newton-Schulz products (`update`).  Norms and answers come alone or, as `norm
train` and `answers train`, with their gradients.  Numbers of nodes, states
and columns are those of the repository's workloads; heads, widths and long
rows are generic.

`own` chooses between the plain forms (elementary torch operations in 32 bits,
in 64 for angles and for sums over all tokens) and the package's operators.
`exact` repeats a pass from the definition in 64 bits and uses nothing of the
package.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZES = {"bf16": 2, "fp16": 2, "fp32": 4}
COEFS = [(3.4445, -4.7750, 2.0315)] * 5
NORM_EPS = 1e-6
UPDATE_EPS = 1e-7
MAX_BYTES = 1.1e9      # the largest listed tensors, read and written
MAX_FLOPS = 1.4e12     # the largest listed update


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # the unknown half of 256 columns of 330 mixed-cardinality nodes (2 to 8 states, padded to 8): every entry's
        # answer with its entropy and the two most likely states
        dict(name="answers of 256 columns", do="answers", rows=42_240, cols=8, stride=8, ragged=True, top=2,
             dtype="fp32"),
        # one entry of very many states, asked for alone: latency
        dict(name="answer of one entry", do="answers", rows=1, cols=32_767, stride=32_767, ragged=False, top=20,
             dtype="bf16"),
        # long rows with many alternatives, in a padded buffer
        dict(name="answers of long rows", do="answers", rows=130, cols=100_003, stride=100_008, ragged=False, top=20,
             dtype="fp16"),
        # training: loss and entropy of the known entries of 2,000 columns of the thousand-node network
        dict(name="answers train nodes", do="answers train", rows=1_200_000, cols=8, stride=8, ragged=True, top=0,
             dtype="fp32"),
        # training with long rows
        dict(name="answers train long", do="answers train", rows=4_099, cols=32_768, stride=32_768, ragged=False,
             top=0, dtype="bf16"),
        # one query and its own key: latency
        dict(name="norm one token", do="norm", q=1, k=1, hq=8, hkv=2, d=64, rot=64, far=20_000, dtype="bf16"),
        # queries and keys of many long columns in one segment, the largest
        dict(name="norm large", do="norm", q=65_536, k=65_536, hq=16, hkv=4, d=128, rot=128, far=65_536, dtype="bf16"),
        # training step of 128 columns of 330 nodes: queries, keys and their gradients, the weights' among them
        dict(name="norm train columns", do="norm train", q=21_120, k=21_120, hq=8, hkv=8, d=64, rot=32, far=128,
             dtype="fp16"),
        # heads of 80, no rotation, no whole cache lines
        dict(name="norm train odd", do="norm train", q=4_099, k=7_951, hq=16, hkv=4, d=80, rot=0, far=1, dtype="fp32"),
        # the imputer's output matrix
        dict(name="update output", do="update", n=1, rows=128, cols=128, dtype="fp32"),
        # its answer matrices, one of 8 states x 128 for each of 1000 nodes
        dict(name="update answers", do="update", n=1_000, rows=8, cols=128, dtype="fp32"),
        # the matrices of a wide network, the largest
        dict(name="update wide", do="update", n=1, rows=4_096, cols=4_096, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, costing no more than the listed."""
    do = rng.choice(["answers", "answers train", "norm", "norm train", "update", "update"])
    while True:
        case = dict(do=do, dtype=rng.choice(["bf16", "fp16", "fp32"]))
        if do.startswith("answers"):
            if rng.random() < 0.5:   # states of nodes
                case.update(rows=_log(rng, 1, 1_200_000), cols=rng.choice([2, 3, 4, 5, 8, 13, 16]),
                            ragged=rng.random() < 0.6)
                top = rng.choice([0, 1, 2])
            else:                    # long rows
                case.update(rows=_log(rng, 1, 20_000), cols=_log(rng, 17, 130_000), ragged=rng.random() < 0.3)
                top = rng.choice([0, 1, 5, 20])
            case.update(stride=case["cols"] + rng.choice([0, 0, 1, 8]),
                        top=min(top, 2 if case["ragged"] else case["cols"]) if do == "answers" else 0)
        elif do.startswith("norm"):
            hkv, d = rng.choice([1, 2, 4, 8]), rng.choice([32, 40, 64, 64, 80, 96, 128, 128])
            case.update(q=_log(rng, 1, 66_000), k=_log(rng, 1, 66_000), hq=hkv * rng.choice([1, 1, 2, 4]), hkv=hkv,
                        d=d, rot=rng.choice([0, d // 2 // 2 * 2, d, d]), far=_log(rng, 2, 1_000_000))
        else:
            case.update(n=_log(rng, 1, 1_000), rows=_log(rng, 1, 4_096), cols=_log(rng, 1, 4_096))
        w = work(case)
        if w["bytes"] <= MAX_BYTES and w["flops"] <= MAX_FLOPS:
            return case


def _counted(case):
    """Logits that count, in the mean."""
    return case["rows"] * ((2 + case["cols"]) / 2 if case["ragged"] else case["cols"])


def work(case):
    size = SIZES[case["dtype"]]
    if case["do"].startswith("answers"):
        rows, logits = case["rows"], _counted(case)
        ends = rows * (4 + (4 if case["ragged"] else 0))       # targets and counts
        if case["do"] == "answers":
            return {"bytes": int(logits * size + ends + rows * (8 + 8 * case["top"])), "flops": int(6 * logits)}
        # values and their gradients a row, the gradient of every logit
        return {"bytes": int(logits * size + case["rows"] * case["cols"] * size + ends + rows * 16),
                "flops": int(12 * logits)}
    if case["do"].startswith("norm"):
        heads = case["q"] * case["hq"] + case["k"] * case["hkv"]
        small = 8 * case["d"] + (4 * (case["q"] + case["k"]) if case["rot"] else 0)
        if case["do"] == "norm":
            return {"bytes": 2 * heads * case["d"] * size + small, "flops": 7 * heads * case["d"]}
        return {"bytes": 4 * heads * case["d"] * size + small + 8 * case["d"], "flops": 19 * heads * case["d"]}
    lo, hi = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
    # X X^T and A A are symmetric: half of each
    return {"bytes": 2 * case["n"] * lo * hi * size, "flops": len(COEFS) * case["n"] * lo * lo * (3 * hi + lo)}


# ----------------------------------------------------------------- the inputs

def _angles(case):
    """Radians a position, of every pair: 10,000^(-2i / rot)."""
    return 10_000.0 ** (-2.0 * np.arange(case["rot"] // 2) / max(case["rot"], 1))


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed((seed * 1_000_003 + 29) % (1 << 62))
    dt = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dt)

    def whole(high, n):
        return torch.randint(0, high, (n,), generator=g, device="cuda").to(torch.int32)

    if case["do"].startswith("answers"):
        rows, cols = case["rows"], case["cols"]
        st = dict(logits=normal(rows, case["stride"], scale=2.5)[:, :cols], counts=None)
        if case["ragged"]:
            st["counts"] = 2 + whole(cols - 1, rows)
            u = torch.rand(rows, generator=g, device="cuda", dtype=torch.float64)
            st["targets"] = torch.minimum((u * st["counts"]).to(torch.int32), st["counts"] - 1)
        else:
            st["targets"] = whole(cols, rows)
        if case["do"] == "answers train":
            # a mean over the rows as the loss, and a little of the entropy
            st["dlogp"] = torch.randn(rows, generator=g, device="cuda") * 0.25 - 1.0
            st["dentropy"] = torch.randn(rows, generator=g, device="cuda") * 0.05
        return st
    if case["do"].startswith("norm"):
        st = dict(q=normal(case["q"], case["hq"], case["d"], scale=1.7),
                  k=normal(case["k"], case["hkv"], case["d"], scale=0.6))
        for side in "qk":
            st["w" + side] = 1.0 + 0.2 * torch.randn(case["d"], generator=g, device="cuda")
            st["pos" + side] = whole(case["far"], case[side]) if case["rot"] else None
            if case["do"] == "norm train":
                st["dout" + side] = normal(*st[side].shape)
        return st
    # a gradient: a few strong directions over noise
    n, rows, cols = case["n"], case["rows"], case["cols"]
    left, right = normal(n, rows, 4).float(), normal(n, 4, cols).float()
    return dict(g=((left[:, :, :, None] * right[:, None]).sum(dim=2) * 3e-4 + 2e-4 * normal(n, rows, cols).float()
                   if rows * cols * n <= 1 << 22 else
                   torch.matmul(left, right) * 3e-4 + 2e-4 * normal(n, rows, cols).float()).to(dt))


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if case["do"].startswith("norm"):
        st["angles"] = _angles(case)
    if not own:
        if case["do"].startswith("norm"):
            st["angles"] = torch.from_numpy(st["angles"]).cuda()
        return st
    import paper_1511_06416_amd as same
    if case["do"].startswith("answers"):
        rows = case["rows"]
        st["logp"], st["entropy"] = (torch.empty(rows, device="cuda") for _ in range(2))
        st["sums"] = torch.empty(rows, 2, device="cuda") if case["do"] == "answers train" else None
        if case["top"]:
            st["top_ids"] = torch.empty(rows, case["top"], dtype=torch.int32, device="cuda")
            st["top_logp"] = torch.empty(rows, case["top"], device="cuda")
        st["ws"] = torch.empty(max(same.same_log_probs_workspace_size(rows, case["cols"], case["top"]), 1),
                               dtype=torch.uint8, device="cuda")
        if case["do"] == "answers train":
            st["dlogits"] = torch.empty(rows, case["cols"], dtype=st["logits"].dtype, device="cuda")
    elif case["do"].startswith("norm"):
        for side in "qk":
            st["out" + side] = torch.empty_like(st[side])
            if case["do"] == "norm train":
                st["d" + side], st["dw" + side] = torch.empty_like(st[side]), torch.empty_like(st["w" + side])
        if case["do"] == "norm train":
            st["ws"] = torch.empty(
                max(same.same_qk_norm_workspace_size(case["d"], case["q"], case["hq"], case["k"], case["hkv"]), 1),
                dtype=torch.uint8, device="cuda")
    else:
        st["out"] = torch.empty_like(st["g"])
        st["ws"] = torch.empty(max(same.same_orthogonalise_workspace_size(*st["g"].shape, st["g"].dtype), 1),
                               dtype=torch.uint8, device="cuda")
    return st


# ------------------------------------------------------------ the plain forms

def _order(x):
    """Whole numbers in the order of fp32 values."""
    bits = x.view(torch.int32).to(torch.int64)
    return torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)


def _plain_answers(st):
    case, x = st["case"], st["logits"].float()
    cols = case["cols"]
    at = torch.arange(cols, device="cuda")
    if st["counts"] is not None:
        x = torch.where(at[None] < st["counts"][:, None], x, float("-inf"))
    target = st["targets"].long()[:, None]
    shifted = x - x.amax(dim=1, keepdim=True)
    e = torch.exp(shifted)
    total = e.sum(dim=1, keepdim=True)
    ls = torch.log(total)
    if st["counts"] is not None:
        shifted = torch.where(at[None] < st["counts"][:, None], shifted, 0.0)   # 0 times e = 0, not -inf times 0
    logp = (shifted.gather(1, target) - ls)[:, 0]
    entropy = (ls - (shifted * e).sum(dim=1, keepdim=True) / total)[:, 0]
    if case["do"] == "answers":
        if not case["top"]:
            return logp, entropy
        # one whole number orders value and place, so that ties go to the lowest index
        key = _order(x) * (1 << 31) - at[None]
        ids = torch.topk(key, case["top"], dim=1).indices
        return logp, entropy, ids.to(torch.int32), x.gather(1, ids) - x.amax(dim=1, keepdim=True) - ls
    p = e / total
    grad = -p * (st["dlogp"][:, None] + st["dentropy"][:, None] * (shifted - ls + entropy[:, None]))
    grad = grad + (at[None] == target) * st["dlogp"][:, None]
    return logp, entropy, grad.to(st["logits"].dtype)


def _turn(case, st, side):
    """Cosines and sines [tokens, 1, rot / 2], from angles in 64 bits."""
    a = st["pos" + side].double()[:, None, None] * st["angles"]
    return torch.cos(a).float(), torch.sin(a).float()


def _plain_norm(st):
    case = st["case"]
    half, outs, grads, weights = case["rot"] // 2, [], [], []
    for side in "qk":
        x = st[side].float()
        dt = st[side].dtype
        r = 1.0 / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + NORM_EPS)
        xhat = x * r
        z = xhat * st["w" + side]
        if half:
            c, s = _turn(case, st, side)
            a, b = z[..., :half], z[..., half:2 * half]
            z = torch.cat([a * c - b * s, b * c + a * s, z[..., 2 * half:]], dim=-1)
        outs.append(z.to(dt))
        if case["do"] == "norm":
            continue
        dz = st["dout" + side].float()
        if half:
            a, b = dz[..., :half], dz[..., half:2 * half]
            dz = torch.cat([a * c + b * s, b * c - a * s, dz[..., 2 * half:]], dim=-1)
        weights.append((dz.double() * xhat.double()).sum(dim=(0, 1)).float())
        dz = dz * st["w" + side]
        grads.append((r * (dz - xhat * (dz * xhat).mean(dim=-1, keepdim=True))).to(dt))
    return tuple(outs + grads + weights)


def _plain_update(st):
    g = st["g"]
    x = g.float()
    tall = g.shape[1] > g.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (torch.sqrt((x * x).sum(dim=(1, 2), keepdim=True)) + UPDATE_EPS)
    for a, b, c in COEFS:
        gram = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    if tall:
        x = x.transpose(1, 2).contiguous()
    return x.to(g.dtype)


# ------------------------------------------------------------------- one pass

def run(state):
    case = state["case"]
    kind = case["do"].split()[0]
    if not own:
        return {"answers": _plain_answers, "norm": _plain_norm, "update": _plain_update}[kind](state)
    import paper_1511_06416_amd as same
    st = state
    if kind == "answers":
        top = case["top"]
        same.same_log_probs(st["logits"], st["targets"], st["logp"], st["ws"], counts=st["counts"], sums=st["sums"],
                            entropy=st["entropy"], top_ids=st["top_ids"] if top else None,
                            top_log_probs=st["top_logp"] if top else None)
        if case["do"] == "answers":
            return (st["logp"], st["entropy"]) + ((st["top_ids"], st["top_logp"]) if top else ())
        same.same_log_probs_backward(st["logits"], st["targets"], st["sums"], st["dlogits"], counts=st["counts"],
                                     entropy=st["entropy"], dlog_probs=st["dlogp"], dentropy=st["dentropy"])
        return st["logp"], st["entropy"], st["dlogits"]
    if kind == "norm":
        args = dict(q_weight=st["wq"], k_weight=st["wk"], q_positions=st["posq"], k_positions=st["posk"],
                    angles=st["angles"], eps=NORM_EPS)
        same.same_qk_norm(st["q"], st["k"], st["outq"], st["outk"], **args)
        if case["do"] == "norm":
            return st["outq"], st["outk"]
        same.same_qk_norm_backward(st["q"], st["k"], st["doutq"], st["doutk"], st["dq"], st["dk"], st["dwq"],
                                   st["dwk"], st["ws"], **args)
        return st["outq"], st["outk"], st["dq"], st["dk"], st["dwq"], st["dwk"]
    same.same_orthogonalise(st["g"], st["out"], st["ws"], coefs=COEFS, eps=UPDATE_EPS)
    return st["out"]


# ---------------------------------------------------------- the 64-bit answer

def _exact_answers(case, st):
    outs = ([], [], [], [])
    step = max(1, (1 << 26) // case["cols"])
    for r in range(0, case["rows"], step):
        part = slice(r, r + step)
        x = st["logits"][part].double()
        if st["counts"] is not None:
            x = x.masked_fill(torch.arange(case["cols"], device="cuda") >= st["counts"][part, None], -math.inf)
        lp = torch.log_softmax(x, dim=1)
        p = lp.exp()
        h = torch.special.entr(p).sum(dim=1)
        t = st["targets"][part].long()
        outs[0].append(lp[torch.arange(len(t), device="cuda"), t])
        outs[1].append(h)
        if case["top"]:
            order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
            outs[2].append(order.to(torch.int32))
            outs[3].append(torch.take_along_dim(lp, order, dim=1))
        elif case["do"] == "answers train":
            dl, dh = st["dlogp"][part, None].double(), st["dentropy"][part, None].double()
            grad = -dl * p - dh * torch.where(p > 0, p * (lp + h[:, None]), 0.0)
            outs[2].append(grad.scatter_add(1, t[:, None], dl))
    return tuple(torch.cat(o) for o in outs if o)


def _exact_norm(case, st):
    outs, grads, weights = [], [], []
    h = case["rot"] // 2
    for side in "qk":
        x, w = st[side].double(), st["w" + side].double()
        norm = (x.square().mean(dim=2) + NORM_EPS).sqrt()[:, :, None]
        z = w * x / norm
        if h:
            turn = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"),
                               st["pos" + side].double()[:, None] * torch.from_numpy(_angles(case)).cuda())[:, None]
            pair = torch.complex(z[:, :, :h].contiguous(), z[:, :, h:2 * h].contiguous()) * turn
            z[:, :, :h], z[:, :, h:2 * h] = pair.real, pair.imag
        outs.append(z)
        if case["do"] == "norm train":
            dz = st["dout" + side].double()
            if h:
                pair = torch.complex(dz[:, :, :h].contiguous(), dz[:, :, h:2 * h].contiguous()) * turn.conj()
                dz[:, :, :h], dz[:, :, h:2 * h] = pair.real, pair.imag
            weights.append((dz * x / norm).sum(dim=0).sum(dim=0))
            u = dz * w
            grads.append(u / norm - x * ((u * x).mean(dim=2)[:, :, None] / norm ** 3))
    return tuple(outs + grads + weights)


def _exact_update(case, st):
    out = []
    step = max(1, (1 << 25) // (case["rows"] * case["cols"]))
    for part in st["g"].double().split(step):
        x = part / (torch.linalg.matrix_norm(part)[:, None, None] + UPDATE_EPS)
        eye = torch.eye(min(case["rows"], case["cols"]), dtype=torch.float64, device="cuda")
        for a, b, c in COEFS:
            # X (a + S (b + c S)) with S = X^T X, or from the left with S = X X^T: the same polynomial
            if case["rows"] >= case["cols"]:
                s = x.mT.contiguous() @ x
                x = x @ (a * eye + s @ (b * eye + c * s))
            else:
                s = x @ x.mT.contiguous()
                x = (a * eye + s @ (b * eye + c * s)) @ x
        out.append(x)
    return torch.cat(out)


def exact(case, seed):
    st = _inputs(case, seed)
    kind = case["do"].split()[0]
    return {"answers": _exact_answers, "norm": _exact_norm, "update": _exact_update}[kind](case, st)
