"""Cases of the path around the grouped products: what is timed, its inputs, its plain form, its exact results.

norm      H = X + R, Y = H w / sqrt(mean H^2 + eps), in the type itself or in 8 bits with a scale for each 128 columns of a row
training  (op "norm_training") the norm and its gradients
round     matrices in 8 bits with a scale for each block of 1 x 128 or 128 x 128
product   Y_g = X_g B_g from 8-bit rows (scales of 1 x 128) and 8-bit matrices (scales of 128 x 128)
route     logits to groups: k choices a row, gates, offsets of the groups, places of the sorted rows, balance loss; and its gradient
rows      rows to their places, the gated sum of what comes back, and the gradients
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E8 = torch.float8_e4m3fn
TOP = 448.0                 # the largest number of 8 bits
LEAST = 2.0 ** -126         # the smallest scale
EPS = 1e-6


def listed():
    return [
        # one new row of one request: latency
        {"name": "norm_token_bf16", "op": "norm", "type": "bf16", "rows": 1, "m": 4096, "residual": True, "eight": True},
        # prompts, in front of a product in 8 bits
        {"name": "norm_prompt_bf16", "op": "norm", "type": "bf16", "rows": 16384, "m": 4096, "residual": True, "eight": True},
        # a training batch, forward and backward
        {"name": "norm_training_bf16", "op": "norm_training", "type": "bf16", "rows": 8192, "m": 4096, "residual": True},
        # the matrices of eight groups, once after each of an optimiser's steps
        {"name": "round_matrices_bf16", "op": "round", "type": "bf16", "count": 8, "rows": 4096, "m": 2048, "block": 128},
        # gradients of a batch on their way to a product in 8 bits, the framework's own type, an odd width
        {"name": "round_rows_f32", "op": "round", "type": "f32", "count": 1, "rows": 3001, "m": 1433, "block": 1},
        # a decode step of a large batch over many groups: a handful of rows each, bound by reading the groups' matrices
        {"name": "product_batch_bf16", "op": "product", "type": "bf16", "groups": 64, "rows": 512, "m": 4096, "n": 2048, "transposed": True},
        # prompts: hundreds of rows for each group
        {"name": "product_prompt_bf16", "op": "product", "type": "bf16", "groups": 16, "rows": 8192, "m": 4096, "n": 4096, "transposed": False},
        # sums as they are, sizes that no tile divides
        {"name": "product_odd_f32", "op": "product", "type": "f32", "groups": 9, "rows": 1237, "m": 515, "n": 389, "transposed": False},
        # one decode step of a few requests
        {"name": "route_decode_f32", "op": "route", "type": "f32", "rows": 24, "groups": 64, "k": 4, "normalise": True, "masked": False, "back": False},
        # a training batch with padding, the balance loss and its gradient
        {"name": "route_training_bf16", "op": "route", "type": "bf16", "rows": 16384, "groups": 128, "k": 8, "normalise": True, "masked": True, "back": True},
        # one decode step: rows to their groups and back
        {"name": "rows_decode_bf16", "op": "rows", "type": "bf16", "rows": 24, "k": 4, "m": 4096, "masked": False, "back": False},
        # a training batch with padding: there, back, and the gradients of both
        {"name": "rows_training_bf16", "op": "rows", "type": "bf16", "rows": 8192, "k": 4, "m": 4096, "masked": True, "back": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    """Operations, and bytes at the rate of 100 operations each."""
    w = work(case)
    return w["flops"] + 100 * w["bytes"]


def _width(rng):
    """Half of the widths are multiples of 64, the others anything."""
    v = _log(rng, 64, 8192)
    return max(64, v // 64 * 64) if rng.random() < 0.5 else v


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["norm", "norm_training", "round", "product", "product", "route", "rows"])
        case = {"op": op, "type": rng.choice(["bf16", "bf16", "f16", "f32"])}
        if op in ("norm", "norm_training"):
            case.update(rows=_log(rng, 1, 16384), m=_width(rng), residual=rng.random() < 0.6)
            if op == "norm":
                case["eight"] = rng.random() < 0.6
        elif op == "round":
            case["block"] = rng.choice([1, 128])
            case.update(count=_log(rng, 1, 16) if case["block"] > 1 else 1, rows=_log(rng, 16, 8192), m=_width(rng))
        elif op == "product":
            case.update(groups=_log(rng, 1, 64), rows=_log(rng, 1, 16384), m=_width(rng), n=_width(rng), transposed=rng.random() < 0.5)
        elif op == "route":
            groups = _log(rng, 2, 512)
            case.update(rows=_log(rng, 1, 65536), groups=groups, k=min(groups, rng.randint(1, 8)), normalise=rng.random() < 0.5,
                        masked=rng.random() < 0.5, back=rng.random() < 0.5)
        else:
            case.update(rows=_log(rng, 1, 16384), k=rng.randint(1, 8), m=_width(rng), masked=rng.random() < 0.5, back=rng.random() < 0.5)
        if _cost(case) <= most:
            return case


def _lengths(total, parts, seed):
    """Ragged lengths that add up to `total`: popular parts and parts that get nothing."""
    rng = np.random.default_rng(seed)
    share = rng.gamma(0.8, size=parts) + 1e-9
    return rng.multinomial(total, share / share.sum()).tolist()


# ---- 8 bits ---------------------------------------------------------------------------

def _eight(x, block):
    """Codes and scales of blocks of `block` x 128 of a stack of matrices; 32 or 64 bits, as x is."""
    count, rows, m = x.shape
    up, left = -rows % block, -m % 128
    x = torch.nn.functional.pad(x, (0, left, 0, up))
    tiles = x.view(count, (rows + up) // block, block, (m + left) // 128, 128)
    scale = (tiles.abs().amax(dim=(2, 4)) / TOP).clamp_min(LEAST)
    codes = (tiles / scale[:, :, None, :, None]).clamp(-TOP, TOP).to(E8)
    return codes.view(count, rows + up, m + left)[:, :rows, :m].contiguous(), scale


def _values(codes, scale, block, dtype):
    """What codes and scales stand for."""
    rows, m = codes.shape[-2:]
    s = scale.to(dtype).repeat_interleave(128, dim=-1)[..., :m]
    if block > 1:
        s = s.repeat_interleave(block, dim=-2)[..., :rows, :]
    return codes.to(dtype) * s


# ---- inputs ----------------------------------------------------------------------------

def prepare(case, seed):
    dt, rows, op = TYPES[case["type"]], case["rows"], case["op"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=dt):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dtype).mul_(scale)

    def empty(*shape, dtype=dt):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    s = {"case": case}
    if op in ("norm", "norm_training"):
        m = case["m"]
        s["X"] = normal(rows, m)
        s["w"] = normal(m, scale=0.2).add_(1.0)
        s["R"] = normal(rows, m, scale=2.0) if case["residual"] else None
        if op == "norm_training":
            s["dY"] = normal(rows, m)
            s["dH"] = normal(rows, m) if case["residual"] else None
        if own:                 # what a serving or training loop allocates once
            s["H"] = empty(rows, m) if case["residual"] else None
            if op == "norm_training":
                s.update(Y=empty(rows, m), rstd=empty(rows, dtype=torch.float32), dX=empty(rows, m), dw=empty(m))
            elif case["eight"]:
                s.update(Y8=empty(rows, m, dtype=E8), scale=empty(rows, -(-m // 128), dtype=torch.float32))
            else:
                s["Y"] = empty(rows, m)
    elif op == "round":
        count, m, b = case["count"], case["m"], case["block"]
        # rows and columns of different sizes, as weights and gradients have
        s["X"] = (normal(count, rows, m) * torch.exp(normal(count, rows, 1)) * torch.exp(normal(1, 1, m))).contiguous()
        if own:
            s.update(X8=empty(count, rows, m, dtype=E8), scale=empty(count, -(-rows // b), -(-m // 128), dtype=torch.float32))
    elif op == "product":
        m, n, t = case["m"], case["n"], case["transposed"]
        lengths = _lengths(rows, case["groups"], seed)
        ends = np.cumsum([0] + lengths)
        s["ends"], s["offsets"] = ends.tolist(), torch.from_numpy(ends.astype(np.int64)).cuda()
        x, xs = _eight(normal(1, rows, m, dtype=torch.float32), 1)
        s["X8"], s["xs"] = x[0], xs[0].contiguous()
        parts = [_eight(normal(1, *((n, m) if t else (m, n)), scale=m ** -0.5, dtype=torch.float32), 128) for _ in range(case["groups"])]
        s["B8"], s["bs"] = torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])
        if own:
            s["Y"] = empty(rows, n)
    elif op == "route":
        G, k = case["groups"], case["k"]
        # popular groups, and rows that are sure of theirs
        l = normal(rows, G, scale=1.5, dtype=torch.float32) + normal(1, G, dtype=torch.float32)
        if case["masked"]:      # groups that a row may not have; the last rows are padding
            l.masked_fill_(torch.rand(rows, G, generator=g, device="cuda") < 0.05, -math.inf)
            l[rows - rows // 16:] = -math.inf
        s["logits"] = l.to(dt)
        if case["back"]:
            s["dgate"], s["dbalance"] = normal(rows, k, dtype=torch.float32), torch.full((1,), 0.01 * rows, device="cuda")
        if own:
            s.update(choice=empty(rows, k, dtype=torch.int32), gate=empty(rows, k, dtype=torch.float32), offsets=empty(G + 1, dtype=torch.int64),
                     place=empty(rows, k, dtype=torch.int32), balance=empty(1, dtype=torch.float32))
            if case["back"]:
                s["dlogits"] = empty(rows, G)
    else:
        k, m = case["k"], case["m"]
        there = torch.rand(rows, k, generator=g, device="cuda") >= (0.05 if case["masked"] else 0.0)
        place = torch.full((rows, k), -1, dtype=torch.int32, device="cuda")
        count = int(there.sum())
        place[there] = torch.randperm(count, generator=g, device="cuda").int()
        s["place"], s["gate"] = place, torch.rand(rows, k, generator=g, device="cuda") / k
        s["X"], s["Z"] = normal(rows, m), normal(rows * k, m)       # rows, and what the groups made of them
        if case["back"]:
            s["dY"], s["dS"] = normal(rows, m), normal(rows * k, m)
        if own:                 # places that nothing has are left as they are
            s.update(S=torch.zeros(rows * k, m, dtype=dt, device="cuda"), Y=empty(rows, m))
            if case["back"]:
                s.update(dZ=torch.zeros(rows * k, m, dtype=dt, device="cuda"), dgate=empty(rows, k, dtype=torch.float32), dX=empty(rows, m))
    return s


# ---- one pass --------------------------------------------------------------------------

def _own(s):
    import paper_2202_09518_amd as nmf
    c = s["case"]
    rows, op = c["rows"], c["op"]
    if op == "norm":
        m = c["m"]
        if c["eight"]:
            nmf.nmf_rms_norm(s["X"], rows, m, EPS, weight=s["w"], R=s["R"], H=s["H"], Y8=s["Y8"], scale=s["scale"])
            return ([s["H"]] if c["residual"] else []) + [s["Y8"], s["scale"]]
        nmf.nmf_rms_norm(s["X"], rows, m, EPS, weight=s["w"], R=s["R"], H=s["H"], Y=s["Y"])
        return ([s["H"]] if c["residual"] else []) + [s["Y"]]
    if op == "norm_training":
        m = c["m"]
        nmf.nmf_rms_norm(s["X"], rows, m, EPS, weight=s["w"], R=s["R"], H=s["H"], Y=s["Y"], rstd=s["rstd"])
        nmf.nmf_rms_norm_gradient(s["H"] if c["residual"] else s["X"], s["rstd"], s["dY"], rows, m, s["dX"], weight=s["w"], dH=s["dH"], dweight=s["dw"])
        return ([s["H"]] if c["residual"] else []) + [s["Y"], s["dX"], s["dw"]]
    if op == "round":
        nmf.nmf_round_blocks(s["X"], rows, c["m"], c["block"], s["X8"], s["scale"])
        return s["X8"], s["scale"]
    if op == "product":
        nmf.nmf_grouped_product8(s["X8"], s["xs"], s["offsets"], c["groups"], rows, s["B8"], s["bs"], c["transposed"], c["m"], c["n"], s["Y"])
        return s["Y"]
    if op == "route":
        G, k = c["groups"], c["k"]
        nmf.nmf_route(s["logits"], rows, G, k, c["normalise"], s["choice"], s["gate"], s["offsets"], s["place"], s["balance"])
        out = [s["choice"], s["gate"], s["offsets"], s["place"], s["balance"]]
        if c["back"]:
            nmf.nmf_route_gradient(s["logits"], rows, G, k, c["normalise"], s["choice"], s["offsets"], s["dgate"], s["dbalance"], s["dlogits"])
            out.append(s["dlogits"])
        return out
    k, m = c["k"], c["m"]
    nmf.nmf_spread_rows(s["X"], rows, k, s["place"], m, s["S"])
    nmf.nmf_collect_rows(s["Z"], rows, k, s["place"], s["gate"], m, s["Y"])
    if not c["back"]:
        return s["S"], s["Y"]
    nmf.nmf_collect_gradient(s["dY"], rows, k, s["place"], s["gate"], m, s["dZ"], X=s["Z"], dgate=s["dgate"])
    nmf.nmf_collect_rows(s["dS"], rows, k, s["place"], None, m, s["dX"])
    return s["S"], s["Y"], s["dZ"], s["dgate"], s["dX"]


def run(state):
    if own:
        return _own(state)
    s, c = state, state["case"]
    rows, op, dt = c["rows"], c["op"], TYPES[c["type"]]
    if op in ("norm", "norm_training"):
        h = s["X"] if s["R"] is None else (s["X"].float() + s["R"].float()).to(dt)
        x = h.float()
        rstd = torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS)
        xhat, w = x * rstd, s["w"].float()
        y = xhat * w
        first = [] if s["R"] is None else [h]
        if op == "norm":
            if c["eight"]:
                codes, scale = _eight(y[None], 1)
                return first + [codes[0], scale[0]]
            return first + [y.to(dt)]
        dy = s["dY"].float()
        z = dy * w
        dx = rstd * (z - xhat * (z * xhat).mean(dim=1, keepdim=True))
        if s["dH"] is not None:
            dx = dx + s["dH"].float()
        return first + [y.to(dt), dx.to(dt), (dy * xhat).sum(dim=0).to(dt)]
    if op == "round":
        return _eight(s["X"].float(), c["block"])
    if op == "product":
        t, ends = c["transposed"], s["ends"]
        X = _values(s["X8"], s["xs"], 1, torch.float32)
        Y = torch.empty(rows, c["n"], dtype=torch.float32, device="cuda")
        for g in range(c["groups"]):
            if ends[g + 1] > ends[g]:
                b = _values(s["B8"][g], s["bs"][g], 128, torch.float32)
                Y[ends[g]:ends[g + 1]] = X[ends[g]:ends[g + 1]] @ (b.t() if t else b)
        return Y.to(dt)
    if op == "route":
        G, k = c["groups"], c["k"]
        l = s["logits"].float()
        top, choice = torch.sort(l, dim=1, descending=True, stable=True)
        chosen = top[:, :k] > -math.inf
        choice = torch.where(chosen, choice[:, :k], -1)
        alive = chosen[:, :1]
        e = torch.where(alive, torch.exp(l - torch.where(alive, top[:, :1], torch.zeros_like(top[:, :1]))), torch.zeros_like(l))
        p = e / torch.where(alive, e.sum(dim=1, keepdim=True), torch.ones_like(top[:, :1]))
        at = choice.clamp_min(0)
        gate = torch.where(chosen, p.gather(1, at), torch.zeros_like(top[:, :k]))
        total = gate.sum(dim=1, keepdim=True)
        part = torch.where(alive, gate / torch.where(alive, total, torch.ones_like(total)), gate)
        if c["normalise"]:
            gate = part
        flat = torch.where(chosen, choice, G).reshape(-1)
        counts = torch.bincount(flat, minlength=G + 1)[:G]
        offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
        order = torch.sort(flat, stable=True).indices
        place = torch.empty_like(order)
        place[order] = torch.arange(rows * k, device="cuda")
        place = torch.where(chosen, place.view(rows, k), -1)
        mine = chosen.sum(dim=1, keepdim=True).double()
        C = counts.sum().clamp_min(1).double()
        q = G * counts.double() / (C * C)
        balance = (q * (mine * p.double()).sum(dim=0)).sum().float().reshape(1)
        out = [choice.int(), gate, offsets, place.int(), balance]
        if c["back"]:
            dg = torch.where(chosen, s["dgate"], torch.zeros_like(gate))
            mean = (dg * gate).sum(dim=1, keepdim=True)
            d = torch.zeros_like(p).scatter_add_(1, at, gate * (dg - mean) if c["normalise"] else gate * dg)
            if not c["normalise"]:
                d = d - p * mean
            q = q.float()
            d = d + s["dbalance"] * mine.float() * p * (q - (p * q).sum(dim=1, keepdim=True))
            out.append(d.to(dt))
        return out
    k, m = c["k"], c["m"]
    place = s["place"].long()
    there = place >= 0
    at, gate = place.clamp_min(0), torch.where(there, s["gate"], torch.zeros_like(s["gate"]))
    row = torch.arange(rows, device="cuda")[:, None].expand(rows, k)[there]
    S = torch.zeros(rows * k, m, dtype=torch.float32, device="cuda")
    S[place[there]] = s["X"].float()[row]
    Z = s["Z"].float()[at]
    Y = (Z * gate[:, :, None]).sum(dim=1)
    if not c["back"]:
        return S.to(dt), Y.to(dt)
    dY = s["dY"].float()
    dZ = torch.zeros(rows * k, m, dtype=torch.float32, device="cuda")
    dZ[place[there]] = (gate[:, :, None] * dY[:, None, :])[there]
    dgate = torch.where(there, (Z * dY[:, None, :]).sum(dim=2), torch.zeros_like(gate))
    dX = (s["dS"].float()[at] * there[:, :, None].float()).sum(dim=1)
    return S.to(dt), Y.to(dt), dZ.to(dt), dgate, dX.to(dt)


def work(case):
    op, rows, e = case["op"], case["rows"], 4 if case["type"] == "f32" else 2
    if op in ("norm", "norm_training"):
        m, n = case["m"], case["rows"] * case["m"]
        r = 1 if case["residual"] else 0
        if op == "norm":
            out = n + 4 * rows * -(-m // 128) if case["eight"] else n * e
            return {"bytes": n * e * (1 + 2 * r) + m * e + out, "flops": 6 * n}
        # X, R and dY, dH read; H, Y, dX and the weight's gradient written; the backward pass reads H (or X) again
        return {"bytes": n * e * (5 + 3 * r) + 2 * m * e, "flops": 16 * n}
    if op == "round":
        n, b = case["count"] * rows * case["m"], case["block"]
        return {"bytes": n * (e + 1) + 4 * case["count"] * -(-rows // b) * -(-case["m"] // 128), "flops": 3 * n}
    if op == "product":
        m, n = case["m"], case["n"]
        used = sum(1 for x in _lengths(rows, case["groups"], 1) if x)
        km, kn = -(-m // 128), -(-n // 128)
        return {"bytes": rows * (m + 4 * km + n * e) + used * (m * n + 4 * km * kn), "flops": 2 * rows * m * n}
    if op == "route":
        G, k = case["groups"], case["k"]
        b = rows * G * e + rows * k * 12 + 8 * (G + 1) + 4
        return {"bytes": b + (2 * rows * G * e + rows * k * 8 if case["back"] else 0), "flops": rows * G * (4 + k) * (2 if case["back"] else 1)}
    k, m = case["k"], case["m"]
    n = rows * m * e
    b = n * (1 + k) + n * (1 + k) + 8 * rows * k
    # dY and Z read, dZ written; dS read, dX written
    return {"bytes": b + (n * (1 + 2 * k) + n * (1 + k) + 8 * rows * k if case["back"] else 0), "flops": rows * m * k * (7 if case["back"] else 2)}


# ---- from the definitions, in 64 bits ----------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    rows, op = case["rows"], case["op"]
    if op in ("norm", "norm_training"):
        h = s["X"].double()
        first = []
        if s["R"] is not None:
            h = (h + s["R"].double()).to(TYPES[case["type"]]).double()      # the norm is that of the row as it is written
            first = [h]
        w = s["w"].double()
        if op == "norm_training":
            h.requires_grad_(True)
            w.requires_grad_(True)
        y = h / (h.square().sum(dim=1, keepdim=True) / case["m"] + EPS).sqrt() * w
        if op == "norm_training":
            y.backward(s["dY"].double())
            dx = h.grad if s["dH"] is None else h.grad + s["dH"].double()
            return [t.detach() for t in first] + [y.detach(), dx, w.grad]
        if not case["eight"]:
            return first + [y]
        codes, scale = _blocks(y, 1)
        return first + [codes, scale]
    if op == "round":
        found = [_blocks(x, case["block"]) for x in s["X"].double()]
        return torch.stack([f[0] for f in found]), torch.stack([f[1] for f in found])
    if op == "product":
        m, n, t = case["m"], case["n"], case["transposed"]
        label = torch.bucketize(torch.arange(rows, device="cuda"), s["offsets"][1:], right=True)
        column = torch.arange(m, device="cuda") // 128
        X = s["X8"].double() * s["xs"].double()[:, column]
        out = X.new_zeros(rows, n)
        for g in range(case["groups"]):
            mine = (label == g).nonzero().squeeze(1)
            if mine.numel() == 0:
                continue
            b = s["B8"][g].double()
            i, j = (torch.arange(z, device="cuda") // 128 for z in b.shape)
            b = b * s["bs"][g].double()[i[:, None], j[None, :]]
            out.index_copy_(0, mine, X.index_select(0, mine) @ (b.t().contiguous() if t else b))
        return out
    if op == "route":
        return _exact_route(case, s)
    k, m = case["k"], case["m"]
    there = s["place"] >= 0
    # the places' own view: which row and which choice each of them has
    t, j = there.nonzero(as_tuple=True)
    z = s["place"][there].long()
    S = torch.zeros(rows * k, m, dtype=torch.float64, device="cuda").index_copy_(0, z, s["X"].double().index_select(0, t))
    weight = s["gate"].double()[t, j][:, None]
    Z = s["Z"].double().index_select(0, z)
    Y = torch.zeros(rows, m, dtype=torch.float64, device="cuda").index_add_(0, t, Z * weight)
    if not case["back"]:
        return S, Y
    dY = s["dY"].double().index_select(0, t)
    dZ = torch.zeros_like(S).index_copy_(0, z, dY * weight)
    dgate = torch.zeros(rows, k, dtype=torch.float64, device="cuda")
    dgate[t, j] = (dY * Z).sum(dim=1)
    dX = torch.zeros_like(Y).index_add_(0, t, s["dS"].double().index_select(0, z))
    return S, Y, dZ, dgate, dX


def _blocks(x, block):
    """8-bit values and scales of one matrix, each entry by the number of its block."""
    rows, m = x.shape
    i, j = torch.arange(rows, device="cuda") // block, torch.arange(m, device="cuda") // 128
    R, M = -(-rows // block), -(-m // 128)
    at = (i[:, None] * M + j[None, :]).reshape(-1)
    most = torch.zeros(R * M, dtype=torch.float64, device="cuda").scatter_reduce_(0, at, x.abs().reshape(-1), "amax")
    scale = (most / TOP).clamp_min(LEAST)
    v = (x.reshape(-1) / scale[at]).clamp(-TOP, TOP)
    # to the nearest of the numbers with three bits behind the leading one, in steps of 2^-9 at least; ties to the even one
    step = torch.exp2((torch.frexp(v).exponent - 4).clamp_min(-9).double())
    return (torch.round(v / step) * step).view(rows, m), scale.view(R, M)


def _exact_route(case, s):
    rows, G, k = case["rows"], case["groups"], case["k"]
    l = s["logits"].double()
    work_l = l.clone()
    choice = torch.full((rows, k), -1, dtype=torch.int64, device="cuda")
    index = torch.arange(G, device="cuda").expand(rows, G)
    for j in range(k):                                       # the largest that is left, the lowest of equals
        most = work_l.amax(dim=1, keepdim=True)
        first = torch.where(work_l == most, index, G).amin(dim=1)
        ok = most.squeeze(1) > -math.inf
        choice[:, j] = torch.where(ok, first, -1)
        work_l.scatter_(1, first[:, None], -math.inf)
    chosen = choice >= 0
    alive = chosen.any(dim=1)
    counts = (choice[:, :, None] == torch.arange(G, device="cuda")).sum(dim=(0, 1)) if rows * k * G < 1 << 28 else \
        torch.stack([(choice == g).sum() for g in range(G)])
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    place = torch.full((rows * k,), -1, dtype=torch.int64, device="cuda")
    for g in range(G):
        mine = (choice.view(-1) == g).nonzero().squeeze(1)
        place[mine] = offsets[g] + torch.arange(mine.numel(), device="cuda")
    some = l[alive].requires_grad_(True)                     # rows that have a choice
    p = torch.softmax(some, dim=1)
    at, ch = choice[alive].clamp_min(0), chosen[alive]
    gates = p.gather(1, at) * ch
    if case["normalise"]:
        gates = gates / gates.sum(dim=1, keepdim=True)
    C = max(1, int(counts.sum()))
    balance = G * (counts.double() / C * (ch.sum(dim=1, keepdim=True) * p / C).sum(dim=0)).sum()
    gate = torch.zeros(rows, k, dtype=torch.float64, device="cuda")
    gate[alive] = gates.detach()
    out = [choice, gate, offsets, place.view(rows, k), balance.detach().reshape(1)]
    if case["back"]:
        d = torch.zeros_like(l)
        if some.numel():
            ((gates * s["dgate"].double()[alive]).sum() + balance * s["dbalance"].double()[0]).backward()
            d[alive] = some.grad
        out.append(d)
    return out
