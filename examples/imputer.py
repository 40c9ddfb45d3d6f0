"""Trains the amortised imputer on partially observed columns of the two-layer
assessment network (30 hidden concepts, 300 items, 90% of the item entries
hidden) and compares its answers for held-out entries with the sampler's.

    python examples/imputer.py [--columns 4000] [--steps 300] [--orthogonal]

Per step a random part of the known entries is hidden (key_mask) and answered
from the rest; the held-out entries are never a key or a target.  The sampler's
figure is that of same_predict after as many steps as asked for.  Both stand
beside the node marginals, which know nothing of the column: on these columns
neither ranks better than they do, so the run compares times and shows the
operators in use, not what an imputer can learn.

With --orthogonal the network norms its queries and keys, the loss comes from
the library's log probabilities, with a little of the entropy as a bonus, and
its matrices take orthogonalised updates.
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_1511_06416_amd as same  # noqa: E402
from paper_1511_06416_amd import evaluate  # noqa: E402
from paper_1511_06416_amd.imputer import Imputer, log_probs  # noqa: E402
from workloads import holdout, make_workload  # noqa: E402


def tokens(entries):
    """Column-major order of a [n][columns] selection: (pointers, nodes, columns)."""
    cols, nodes = np.nonzero(entries.T)
    return np.concatenate([[0], np.cumsum(entries.sum(axis=0))]).astype(np.int64), nodes, cols


def marginals(w):
    """AUC of the held-out entries when every node answers with the share of
    ones among its known entries, whatever the column."""
    obs, target = holdout(w, 0, 0.2)
    cols = w.mb_cols(0)
    known = obs[:, :cols] == 1
    states = w.states[0][:, 0, :cols].cpu().numpy()
    share = ((states == 1) & known).sum(axis=1) + 1.0
    share /= known.sum(axis=1) + 2.0
    _, nodes, columns = tokens(target[:, :cols] >= 0)
    return evaluate.auc(share[nodes], states[nodes, columns] == 1)


def train_imputer(w, steps, drop=0.1, hide=0.3, lr=3e-3, seed=5, orthogonal=False):
    """Returns (AUC of the held-out entries, seconds per step, seconds of the answer)."""
    obs, target = holdout(w, 0, 0.2)
    cols = w.mb_cols(0)
    known = obs[:, :cols] == 1
    test = target[:, :cols] >= 0
    states = w.states[0][:, 0, :cols].cpu().numpy()
    k_ptr, k_node, k_col = tokens(known)
    t_ptr, t_node, t_col = tokens(test)
    key = [torch.from_numpy(x).cuda() for x in (k_node, states[k_node, k_col].astype(np.int64))]
    asked = torch.from_numpy(t_node).cuda()
    torch.manual_seed(seed)
    net = Imputer(w.net.n, int(w.net.card.max()), norm=orthogonal).cuda()
    opts = net.optimisers(other_lr=lr) if orthogonal else (torch.optim.Adam(net.parameters(), lr=lr),)
    card = torch.as_tensor(w.net.card, dtype=torch.int32, device="cuda")
    states32, counts = key[1].to(torch.int32), card[key[0]]
    # training answers known entries, the test held-out ones, from the same keys
    plan = same.same_cross_create(k_ptr, k_ptr, net.heads, net.heads, net.head_dim, net.dtype)
    ask = same.same_cross_create(t_ptr, k_ptr, net.heads, net.heads, net.head_dim, net.dtype)
    ws, ask_ws = plan.new_workspace(backward=True), ask.new_workspace(backward=True)

    def step(s):
        shown = torch.rand(len(k_node), device="cuda") >= hide
        logits = net(plan, ws, key[0], key[0], key[1], key_mask=shown, drop=drop, seed=seed, call_id=s)
        if orthogonal:   # entries that were shown are not asked for
            asked_now = torch.where(shown, -1, states32)
            lp, entropy, _, _ = log_probs(logits, asked_now, counts)
            loss = -(lp.sum() + 0.01 * (entropy * ~shown).sum()) / (~shown).sum()
        else:
            loss = torch.nn.functional.cross_entropy(logits[~shown], key[1][~shown])
        for opt in opts:
            opt.zero_grad(set_to_none=True)
        loss.backward()
        for opt in opts:
            opt.step()
        return loss

    def answer():
        with torch.no_grad():
            logits = net(ask, ask_ws, asked, key[0], key[1])
            if orthogonal:
                return log_probs(logits, torch.ones_like(asked, dtype=torch.int32), card[asked])[0].exp()
            return logits.softmax(dim=1)[:, 1]

    step(0)
    answer()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for s in range(1, steps):
        step(s)
    torch.cuda.synchronize()
    t1 = time.perf_counter()
    p = answer().cpu().numpy()
    t2 = time.perf_counter()
    return evaluate.auc(p, states[t_node, t_col] == 1), (t1 - t0) / max(steps - 1, 1), t2 - t1


def train_sampler(w, steps, sweeps=20):
    """AUC of same_predict's answers for the same entries."""
    obs, target = holdout(w, 0, 0.2)
    pptr, pidx, card = w.net.csr()
    ctx = same.same_create(pptr, pidx, card, w.alpha)
    ws = ctx.new_workspace()
    st, ob = same.pack_states(w.states[0]).cuda(), torch.from_numpy(obs).cuda()
    cpts = torch.from_numpy(w.init_theta).cuda()
    mb, tot = (torch.zeros(ctx.cpt_total, dtype=torch.int32, device="cuda") for _ in range(2))
    same.same_init_latent(ctx, st, ob, w.m, w.n_cols, w.ld, 0, w.seed + 17)
    same.same_counts(ctx, st, w.m, w.n_cols, w.ld, mb, tot, ws)
    for s in range(steps):
        same.same_step(ctx, st, ob, cpts, w.m, w.n_cols, w.ld, 0, w.seed, s, mb, tot, s, ws)
    hits = torch.zeros(target.shape, dtype=torch.int32, device="cuda")
    tgt = torch.from_numpy(target).cuda()
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    same.same_predict(ctx, st, ob, cpts, tgt, w.m, w.n_cols, w.ld, 0, w.seed, steps, sweeps, hits, ws)
    torch.cuda.synchronize()
    seconds = time.perf_counter() - t0
    auc = evaluate.auc(*evaluate.binary_scores(hits.cpu().numpy(), target, sweeps * w.m))
    ctx.close()
    return auc, seconds


def main():
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--columns", type=int, default=4_000)
    a.add_argument("--steps", type=int, default=300)
    a.add_argument("--orthogonal", action="store_true")
    args = a.parse_args()
    w = make_workload(4, n_cols=args.columns)
    print("node marginals: held-out AUC %.4f" % marginals(w))
    auc, per_step, ans = train_imputer(w, args.steps, orthogonal=args.orthogonal)
    print("imputer: held-out AUC %.4f after %d steps of %.2f ms; the answers in %.2f ms"
          % (auc, args.steps, 1e3 * per_step, 1e3 * ans))
    auc, ans = train_sampler(w, args.steps)
    print("sampler: held-out AUC %.4f after %d steps; the answers (20 sweeps) in %.2f ms" % (auc, args.steps, 1e3 * ans))


if __name__ == "__main__":
    main()
