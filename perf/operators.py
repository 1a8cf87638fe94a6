"""Cases of the grouped products and the low-rank adapters: what is timed, its inputs, its plain form, its exact results.

Grouped product:   Y_g = X_g B_g for the rows of each group g, B_g stored as m x n or, `transposed`, as n x m.
Its gradients:     dX_g = dY_g B_g^T and dB_g = X_g^T dY_g (in the layout of B_g).
Low-rank adapters: Y = X A + s_r (X W_r) H_r, r the run (factor pair) of the row's segment, or no run.
Training step:     the forward pass, dX, and the gradients of all W_r and H_r.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # one decode step of a few requests, each row routed to one of 16 groups, some of which get none
        {"name": "product_decode_bf16", "op": "product", "type": "bf16", "groups": 16, "rows": 24, "m": 2048, "n": 2048, "transposed": True},
        # a decode step of a large batch over many groups: a handful of rows each, bound by reading the groups' matrices
        {"name": "product_batch_f16", "op": "product", "type": "f16", "groups": 64, "rows": 512, "m": 4096, "n": 2048, "transposed": False},
        # prompts: hundreds of rows for each group
        {"name": "product_prompt_bf16", "op": "product", "type": "bf16", "groups": 16, "rows": 8192, "m": 4096, "n": 4096, "transposed": False},
        # the framework's own type, sizes that no tile divides
        {"name": "product_odd_f32", "op": "product", "type": "f32", "groups": 9, "rows": 1237, "m": 515, "n": 389, "transposed": False},
        # backward pass of a training batch
        {"name": "gradient_bf16", "op": "gradient", "type": "bf16", "groups": 8, "rows": 8192, "m": 4096, "n": 2048, "transposed": False},
        # backward pass in the framework's own type, odd row count
        {"name": "gradient_f32", "op": "gradient", "type": "f32", "groups": 5, "rows": 1999, "m": 1000, "n": 720, "transposed": True},
        # one new row of one request: latency
        {"name": "adapters_token_bf16", "op": "adapters", "type": "bf16", "rows": 1, "segments": 1, "runs": 8, "kmin": 16, "kmax": 16, "m": 2048, "n": 2048, "transposed": True},
        # one new row for each of 48 requests, ranks of the ensemble's sweep
        {"name": "adapters_decode_bf16", "op": "adapters", "type": "bf16", "rows": 48, "segments": 48, "runs": 15, "kmin": 2, "kmax": 16, "m": 4096, "n": 4096, "transposed": True},
        # short continuations of many requests, A as the framework keeps it
        {"name": "adapters_batch_f16", "op": "adapters", "type": "f16", "rows": 160, "segments": 40, "runs": 24, "kmin": 8, "kmax": 64, "m": 8192, "n": 4096, "transposed": False},
        # long prompts of a few requests
        {"name": "adapters_prompt_bf16", "op": "adapters", "type": "bf16", "rows": 16384, "segments": 11, "runs": 8, "kmin": 8, "kmax": 64, "m": 4096, "n": 4096, "transposed": True},
        # a training step of the factors of several runs
        {"name": "training_bf16", "op": "training", "type": "bf16", "rows": 8192, "segments": 6, "runs": 4, "kmin": 16, "kmax": 64, "m": 4096, "n": 4096, "transposed": False},
        # the same in the framework's own type, ranks of the ensemble's sweep
        {"name": "training_f32", "op": "training", "type": "f32", "rows": 4096, "segments": 15, "runs": 15, "kmin": 2, "kmax": 16, "m": 4096, "n": 2048, "transposed": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    """Operations, those of the 32-bit type counted eight times, and bytes at the rate of 100 operations each."""
    w = work(case)
    return w["flops"] * (8 if case["type"] == "f32" else 1) + 100 * w["bytes"]


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["product", "product", "gradient", "adapters", "adapters", "training"])
        case = {"op": op, "type": rng.choice(["bf16", "bf16", "f16", "f32"]), "transposed": rng.random() < 0.5}
        served = op in ("product", "adapters")
        case["rows"] = _log(rng, 1 if served else 64, 16384)
        # half of the widths are multiples of 64, the others anything
        for d in ("m", "n"):
            v = _log(rng, 128, 8192)
            case[d] = max(64, v // 64 * 64) if rng.random() < 0.5 else v
        if op in ("product", "gradient"):
            case["groups"] = _log(rng, 1, 64)
        else:
            case["segments"] = min(case["rows"], _log(rng, 1, 64))
            case["runs"] = _log(rng, 1, 32)
            case["kmax"] = _log(rng, 4, 64)
            case["kmin"] = rng.randint(1, case["kmax"])
        if _cost(case) <= most and 3072 not in (case["rows"], case["m"], case["n"]):
            return case


def _lengths(total, parts, rng):
    """Ragged lengths that add up to `total`: popular parts and parts that get nothing."""
    share = rng.gamma(0.8, size=parts) + 1e-9
    return rng.multinomial(total, share / share.sum()).tolist()


def _plan(case, seed):
    """Lengths, runs and ranks of a case: host values, from the seed alone."""
    rng = np.random.default_rng([seed, 7])
    if "groups" in case:
        return _lengths(case["rows"], case["groups"], rng), None, None
    if case["segments"] == case["rows"]:
        lengths = [1] * case["rows"]
    else:
        lengths = _lengths(case["rows"], case["segments"], rng)
    runs = rng.integers(0, case["runs"], size=case["segments"]).tolist()
    if case["segments"] >= 8:
        runs[int(rng.integers(0, case["segments"]))] = -1          # a request without an adapter
    lo, hi = case["kmin"], case["kmax"]
    ranks = [lo + (hi - lo) * r // max(1, case["runs"] - 1) for r in range(case["runs"])]
    return lengths, runs, ranks


def prepare(case, seed):
    lengths, runs, ranks = _plan(case, seed)
    dt, m, n, rows = TYPES[case["type"]], case["m"], case["n"], case["rows"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, scale=1.0):
        t = torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32 if dt == torch.float32 else dt)
        return t.mul_(scale)

    ends = np.cumsum([0] + lengths)
    s = {"case": case, "ends": ends.tolist(), "offsets": torch.from_numpy(ends.astype(np.int64)).cuda(), "X": normal(rows, m)}
    shape = (n, m) if case["transposed"] else (m, n)
    if "groups" in case:
        s["B"] = normal(case["groups"], *shape, scale=m ** -0.5)
    else:
        koff = np.cumsum([0] + ranks)
        s.update(A=normal(*shape, scale=m ** -0.5), runs=runs, koff_host=koff.tolist(),
                 run=torch.tensor(runs, dtype=torch.int32, device="cuda"), koff=torch.from_numpy(koff.astype(np.int32)).cuda(),
                 Wt=normal(int(koff[-1]), m, scale=m ** -0.5), H=normal(int(koff[-1]), n, scale=0.5),
                 scale=torch.tensor([2.0 / k for k in ranks], dtype=torch.float32, device="cuda"),
                 scale_host=[float(np.float32(2.0 / k)) for k in ranks])
    if case["op"] in ("gradient", "training"):
        s["dY"] = normal(rows, n)
    if own:
        # what a serving or training loop allocates once
        if case["op"] == "gradient":
            s["dX"], s["dB"] = torch.empty_like(s["X"]), torch.empty_like(s["B"])
        else:
            s["Y"] = torch.empty(rows, n, dtype=dt, device="cuda")
        if case["op"] in ("adapters", "training"):
            s["U"] = torch.empty(rows, case["kmax"], dtype=torch.float32, device="cuda")
        if case["op"] == "training":
            s["V"] = torch.empty_like(s["U"])
            s["dX"], s["dWt"], s["dH"] = torch.empty_like(s["X"]), torch.empty_like(s["Wt"]), torch.empty_like(s["H"])
    return s


def _own(s):
    import paper_2202_09518_amd as nmf
    c = s["case"]
    rows, m, n, t = c["rows"], c["m"], c["n"], c["transposed"]
    if c["op"] == "product":
        nmf.nmf_grouped_product(s["X"], s["offsets"], c["groups"], rows, s["B"], t, m, n, s["Y"])
        return s["Y"]
    if c["op"] == "gradient":
        nmf.nmf_grouped_product(s["dY"], s["offsets"], c["groups"], rows, s["B"], not t, n, m, s["dX"])
        if t:
            nmf.nmf_grouped_gradient(s["dY"], s["X"], s["offsets"], c["groups"], rows, n, m, s["dB"])
        else:
            nmf.nmf_grouped_gradient(s["X"], s["dY"], s["offsets"], c["groups"], rows, m, n, s["dB"])
        return s["dX"], s["dB"]
    nmf.nmf_lowrank_product(s["X"], rows, s["A"], t, m, n, s["offsets"], s["run"], c["segments"], s["Wt"], s["H"], s["koff"], c["runs"],
                            c["kmax"], s["scale"], s["U"], s["Y"])
    if c["op"] == "adapters":
        return s["Y"]
    nmf.nmf_lowrank_product(s["dY"], rows, s["A"], not t, n, m, s["offsets"], s["run"], c["segments"], s["H"], s["Wt"], s["koff"], c["runs"],
                            c["kmax"], s["scale"], s["V"], s["dX"])
    nmf.nmf_lowrank_gradient(s["X"], s["dY"], rows, m, n, s["offsets"], s["run"], c["segments"], s["koff"], c["runs"], c["kmax"],
                             s["U"], s["V"], s["dWt"], s["dH"])
    return s["Y"], s["dX"], s["dWt"], s["dH"]


def run(state):
    if own:
        return _own(state)
    s, c = state, state["case"]
    t, ends, dt = c["transposed"], state["ends"], TYPES[c["type"]]
    X = s["X"].float()
    if "groups" in c:
        B = s["B"]
        if c["op"] == "product":
            Y = torch.empty(c["rows"], c["n"], dtype=torch.float32, device="cuda")
            for g in range(c["groups"]):
                if ends[g + 1] > ends[g]:
                    b = B[g].float()
                    Y[ends[g]:ends[g + 1]] = X[ends[g]:ends[g + 1]] @ (b.t() if t else b)
            return Y.to(dt)
        dY, dX, dB = s["dY"].float(), torch.empty_like(X), torch.zeros(B.shape, dtype=torch.float32, device="cuda")
        for g in range(c["groups"]):
            if ends[g + 1] > ends[g]:
                b, x, dy = B[g].float(), X[ends[g]:ends[g + 1]], dY[ends[g]:ends[g + 1]]
                dX[ends[g]:ends[g + 1]] = dy @ (b if t else b.t())
                dB[g] = dy.t() @ x if t else x.t() @ dy
        return dX.to(dt), dB.to(dt)
    A, Wt, H, koff = s["A"].float(), s["Wt"].float(), s["H"].float(), s["koff_host"]
    Y = X @ (A.t() if t else A)
    back = c["op"] == "training"
    if back:
        dY = s["dY"].float()
        dX = dY @ (A if t else A.t())
        dWt, dH = torch.zeros_like(Wt), torch.zeros_like(H)
    for i, r in enumerate(s["runs"]):
        if r < 0 or ends[i + 1] == ends[i]:
            continue
        rows, k = slice(ends[i], ends[i + 1]), slice(koff[r], koff[r + 1])
        u = (X[rows] @ Wt[k].t()) * s["scale"][r]
        Y[rows] += u @ H[k]
        if back:
            v = (dY[rows] @ H[k].t()) * s["scale"][r]
            dX[rows] += v @ Wt[k]
            dWt[k] += v.t() @ X[rows]
            dH[k] += u.t() @ dY[rows]
    if back:
        return Y.to(dt), dX.to(dt), dWt.to(dt), dH.to(dt)
    return Y.to(dt)


def work(case):
    lengths, runs, ranks = _plan(case, 1)
    m, n, rows, e = case["m"], case["n"], case["rows"], 4 if case["type"] == "f32" else 2
    if "groups" in case:
        used = sum(1 for x in lengths if x)
        if case["op"] == "product":
            return {"bytes": (rows * (m + n) + used * m * n) * e, "flops": 2 * rows * m * n}
        # X, dY and B once; dX and all of dB
        return {"bytes": (rows * (2 * m + n) + (used + case["groups"]) * m * n) * e, "flops": 4 * rows * m * n}
    seen = {r for r, x in zip(runs, lengths) if r >= 0 and x}
    factors = sum(ranks[r] for r in seen) * (m + n)
    low = sum(x * ranks[r] for r, x in zip(runs, lengths) if r >= 0) * 2 * (m + n)
    if case["op"] == "adapters":
        return {"bytes": (rows * (m + n) + m * n + factors) * e, "flops": 2 * rows * m * n + low}
    # X, dY, A and the factors once; Y, dX and the gradients of all factors
    return {"bytes": (2 * rows * (m + n) + m * n + factors + sum(ranks) * (m + n)) * e, "flops": 4 * rows * m * n + 3 * low}


def exact(case, seed):
    """From the definitions, in 64 bits: rows are picked by the number of their group or run, not by ranges."""
    s = prepare(case, seed)
    t = case["transposed"]
    label = torch.bucketize(torch.arange(case["rows"], device="cuda"), s["offsets"][1:], right=True)
    X = s["X"].double()
    if "groups" in case:
        out = X.new_zeros(case["rows"], case["n"])
        grads = case["op"] == "gradient"
        if grads:
            dY, dX, dB = s["dY"].double(), torch.zeros_like(X), []
        for g in range(case["groups"]):
            mine = (label == g).nonzero().squeeze(1)
            b = s["B"][g].double()
            b = b.t().contiguous() if t else b
            if not grads:
                out.index_copy_(0, mine, X.index_select(0, mine) @ b)
                continue
            x, dy = X.index_select(0, mine), dY.index_select(0, mine)
            dX.index_copy_(0, mine, dy @ b.t())
            db = x.t() @ dy
            dB.append(db.t().contiguous() if t else db)
        return (dX, torch.stack(dB)) if grads else out
    A = s["A"].double()
    A = A.t().contiguous() if t else A
    run = torch.tensor(s["runs"], device="cuda")[label]
    W, H = s["Wt"].double().t().contiguous(), s["H"].double()
    back = case["op"] == "training"
    Y = X @ A
    if back:
        dY = s["dY"].double()
        dX, dW, dH = dY @ A.t(), torch.zeros_like(W), torch.zeros_like(H)
    for r in range(case["runs"]):
        mine = (run == r).nonzero().squeeze(1)
        a, b, scale = s["koff_host"][r], s["koff_host"][r + 1], s["scale_host"][r]
        x, w, h = X.index_select(0, mine), W[:, a:b], H[a:b]
        delta = (w @ h) * scale
        Y.index_add_(0, mine, x @ delta)
        if back:
            dy = dY.index_select(0, mine)
            dX.index_add_(0, mine, dy @ delta.t())
            g = (x.t() @ dy) * scale                 # gradient of the whole m x n product W_r H_r
            dW[:, a:b] = g @ h.t()
            dH[a:b] = w.t() @ g
    return (Y, dX, dW.t().contiguous(), dH) if back else Y
