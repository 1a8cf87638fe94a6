"""From an ensemble to its use: learn factor pairs, serve requests of many tasks at once, refine the pairs by their gradients.

Every task r has a map A + D_r: a matrix A that all share and a non-negative change D_r of its own.

1. `nmf_mu_dense_batched` learns D_r ~= W_r H_r, one run for each task, ranks of its own.
2. `nmf_lowrank_product` serves a batch of requests, each a few rows of one task:  Y = X A + X W_r H_r.
3. `nmf_grouped_product` gives the same with the tasks' whole matrices, Y = X (A + D_r): what the pairs are held against.
4. `nmf_lowrank_product` backwards and `nmf_lowrank_gradient` refine W_r and H_r on the requests; `nmf_grouped_gradient`
   gives the gradient that the whole matrices would have had.

    python examples/serve_and_refine.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2202_09518_amd as nmf  # noqa: E402

EPS = 1e-16


def learn(D, ranks, iters, g):
    """Factor pairs of the tasks' changes: Wt (all W_r transposed, one below the other), H and the ranks' offsets."""
    tasks, m, n = D.shape
    W = [torch.rand(m, k, generator=g, device="cuda") for k in ranks]
    H = [torch.rand(k, n, generator=g, device="cuda") for k in ranks]
    nmf.nmf_mu_dense_batched(tasks, [D[r] for r in range(tasks)], m, n, ranks, W, H, iters, EPS)
    koff = torch.tensor([sum(ranks[:r]) for r in range(tasks + 1)], dtype=torch.int32, device="cuda")
    return torch.cat([w.t() for w in W]).contiguous(), torch.cat(H).contiguous(), koff


def run(m=512, n=384, tasks=5, requests=12, iters=60, steps=20, seed=1, verbose=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    A = torch.randn(m, n, generator=g, device="cuda") / m ** 0.5
    ranks = [2 + 2 * r for r in range(tasks)]
    D = torch.stack([torch.rand(m, 6, generator=g, device="cuda") @ torch.rand(6, n, generator=g, device="cuda") for _ in range(tasks)]) / m
    Wt, H, koff = learn(D, ranks, iters, g)
    kmax = max(ranks)

    # requests of 1 to 40 rows, each of some task, sorted by task so that the tasks' whole matrices can be grouped
    lengths = torch.randint(1, 41, (requests,), generator=g, device="cuda")
    task = torch.randint(0, tasks, (requests,), generator=g, device="cuda").sort().values.int()
    offsets = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)])
    rows = int(offsets[-1])
    of_row = torch.repeat_interleave(task.long(), lengths)
    bounds = torch.searchsorted(of_row, torch.arange(tasks + 1, device="cuda"))
    X = torch.randn(rows, m, generator=g, device="cuda")

    whole = (A + D).contiguous()
    target = torch.empty(rows, n, device="cuda")
    nmf.nmf_grouped_product(X, bounds, tasks, rows, whole, False, m, n, target)

    Y, dX = torch.empty_like(target), torch.empty_like(X)
    U, V = torch.empty(rows, kmax, device="cuda"), torch.empty(rows, kmax, device="cuda")
    dWt, dH = torch.empty_like(Wt), torch.empty_like(H)

    def serve(Wt, H):
        nmf.nmf_lowrank_product(X, rows, A, False, m, n, offsets, task, requests, Wt, H, koff, tasks, kmax, None, U, Y)
        return float((Y - target).square().sum() / target.square().sum())

    def gradients():
        dY = (Y - target) / rows
        nmf.nmf_lowrank_product(dY, rows, A, True, n, m, offsets, task, requests, H, Wt, koff, tasks, kmax, None, V, dX)
        nmf.nmf_lowrank_gradient(X, dY, rows, m, n, offsets, task, requests, koff, tasks, kmax, U, V, dWt, dH)
        return dY

    losses = [serve(Wt, H)]
    rate = 1.0
    for _ in range(steps):
        gradients()
        while True:                                  # along the gradients, shorter until it helps
            Wn, Hn = Wt - rate * dWt, H - rate * dH
            loss = serve(Wn, Hn)
            if loss < losses[-1] or rate < 1e-12:
                break
            rate *= 0.25
        if loss >= losses[-1]:
            break
        Wt, H, rate = Wn, Hn, rate * 2
        losses.append(loss)
    losses.append(serve(Wt, H))
    dY = gradients()
    # the whole matrices' gradient at the same point: the pairs' are its products with them
    G = torch.empty(tasks, m, n, device="cuda")
    nmf.nmf_grouped_gradient(X, dY, bounds, tasks, rows, m, n, G)
    off = 0.0
    for r in range(tasks):
        k = slice(int(koff[r]), int(koff[r + 1]))
        want = H[k].double() @ G[r].double().t()
        off = max(off, float((dWt[k].double() - want).norm() / want.norm().clamp_min(1e-30)) if float(want.norm()) else 0.0)
    if verbose:
        print(f"{requests} requests of {tasks} tasks, {rows} rows, ranks {ranks}")
        print("relative squared error of the served rows:", " ".join(f"{x:.3e}" for x in losses[::5]))
        print(f"gradients of the pairs against the whole matrices': {off:.1e}")
    return losses, off


if __name__ == "__main__":
    run()
