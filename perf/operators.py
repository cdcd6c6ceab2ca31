"""Performance cases of the operators that stand between the residual stream and the experts.

Four operators, each with its gradient:

  sort    tokens to their experts: from the choice `ids` [T, k] the plan (rows of every expert in token order, where each
          pair's row is) and the tokens' copies in it;                   backward: dX of the copies' gradients
  unsort  the experts' rows back in token order, weighted and summed;    backward: gradients of the rows and of the weights
  norm    the norm before a block, x / sqrt(mean x^2 + eps) * w;         backward: dX, with the gradient that comes along
          the residual added, and dw
  join    behind a block: its output normed, gated, scaled and added to the scaled residual, and the next block's norm
          of the sum;                                                    backward: all five gradients

Keys of a case: op, direction "forward" or "backward", T tokens, d hidden size, dtype "bf16" or "f32"; for sort and unsort
E experts, k experts per token, align (rows of an expert start at a multiple of it; no pair is dropped) or capacity (above 0:
the layer's own buffers, rows of expert e from e * roundup(capacity, 128) on, later pairs dropped), lost (share of tokens without an
expert: padding), skew (spread of the experts' popularity); for join gate (a factor per token), post (norm behind the
block) and next (the next block's norm in the same call).
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
RES_SCALE, BRANCH_SCALE = 0.875, 0.5


def _rows_case(name, op, direction, T, d, E, k, dtype="bf16", align=1, capacity=0, lost=0.0, skew=1.0):
    return {"name": name, "op": op, "direction": direction, "T": T, "d": d, "E": E, "k": k, "dtype": dtype, "align": align,
            "capacity": capacity, "lost": lost, "skew": skew}


def _norm_case(name, op, direction, T, d, dtype="bf16", gate=False, post=True, next_norm=True):
    c = {"name": name, "op": op, "direction": direction, "T": T, "d": d, "dtype": dtype}
    return dict(c, gate=gate, post=post, next=next_norm) if op == "join" else c


def listed():
    return [
        # A decode step of a serving batch: the choice of 64 tokens among the small layer's 16 experts.
        _rows_case("sort_decode", "sort", "forward", T=64, d=1024, E=16, k=2),
        # A training step in the layer's capacity-bounded buffers, 1.25 times the even load, on a skewed choice.
        _rows_case("sort_capacity", "sort", "forward", T=16384, d=2048, E=32, k=2, align=128, capacity=1280),
        # The largest batch, nothing dropped, every expert's rows starting at a tile of 128.
        _rows_case("sort_large", "sort", "forward", T=65536, d=4096, E=64, k=2, align=128),
        # Gradient of an fp32 batch with odd sizes and three experts per token, a part of it padding.
        _rows_case("sort_backward_ragged_f32", "sort", "backward", T=3001, d=1088, E=12, k=3, dtype="f32", lost=0.1),
        # A decode step of a layer of many narrow experts, eight per token.
        _rows_case("unsort_decode", "unsort", "forward", T=64, d=2048, E=128, k=8),
        # A ragged prefill batch of that layer, a part of it padding.
        _rows_case("unsort_prefill", "unsort", "forward", T=6113, d=2048, E=128, k=8, lost=0.05),
        # A mid-sized model's training step.
        _rows_case("unsort_backward", "unsort", "backward", T=16384, d=2048, E=32, k=2),
        # The norm of an fp32 batch whose sizes are no powers of two.
        _norm_case("norm_ragged_f32", "norm", "forward", T=1531, d=768, dtype="f32"),
        # Its gradient in a mid-sized model's training step.
        _norm_case("norm_backward", "norm", "backward", T=16384, d=2048),
        # A decode step: the block's output joins the residual, and the next block's norm follows.
        _norm_case("join_decode", "join", "forward", T=64, d=4096),
        # A ragged prefill batch with a gate per token.
        _norm_case("join_prefill", "join", "forward", T=6113, d=2048, gate=True),
        # The largest training step.
        _norm_case("join_backward_large", "join", "backward", T=65536, d=4096, gate=True),
    ]


def draw(rng):
    """T from 1 to 65536, d from 64 to 8192, E from 2 to 256, k from 1 to 8, all layouts, directions and types."""
    op = rng.choice(("sort", "unsort", "norm", "join"))
    direction = rng.choice(("forward", "backward"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    b = 2 if dtype == "bf16" else 4
    d = 8 * max(8, min(1024, round(math.exp(rng.uniform(math.log(8), math.log(1024))))))
    T = max(1, round(math.exp(rng.uniform(0.0, math.log(65536)))))
    if op in ("norm", "join"):
        T = max(1, min(T, 65536 * 4096 * 2 // (d * b)))
        return _norm_case("", op, direction, T, d, dtype, rng.random() < 0.5, rng.random() < 0.75, rng.random() < 0.75)
    E = max(2, min(256, round(math.exp(rng.uniform(math.log(2), math.log(256))))))
    k = rng.randint(1, min(8, E))
    T = max(1, min(T, 65536 * 4096 * 2 * 2 // (d * b * k)))
    capacity = math.ceil(rng.uniform(0.5, 1.5) * T * k / E) if rng.random() < 0.3 else 0
    align = 128 if capacity else rng.choice((1, 8, 128))
    return _rows_case("", op, direction, T, d, E, k, dtype, align, capacity, rng.choice((0.0, 0.0, 0.1)), rng.uniform(0.0, 2.0))


# ---- inputs ----------------------------------------------------------------------------------


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _n_rows(c):
    """Rows of the buffers that hold the sorted tokens."""
    if c["capacity"]:
        return c["E"] * ((c["capacity"] + 127) // 128 * 128)
    n = c["T"] * c["k"]
    return n + min(c["E"], n) * (c["align"] - 1)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    T, d, dt = c["T"], c["d"], _dtype(c)

    def normal(*shape, dtype=dt, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda", dtype=dtype if dtype == torch.float32 else torch.bfloat16) * scale).to(dtype)

    def empty(*shape, dtype=dt):
        return torch.zeros(*shape, device="cuda", dtype=dtype)

    s = {"c": c}
    if c["op"] in ("sort", "unsort"):
        E, k, R = c["E"], c["k"], _n_rows(c)
        score = torch.randn(T, E, generator=g, device="cuda") + c["skew"] * torch.randn(E, generator=g, device="cuda")
        top = torch.topk(score, k, dim=1)
        ids = top.indices.to(torch.int32)
        ids[torch.rand(T, generator=g, device="cuda") < c["lost"]] = -1
        s["ids"] = ids.contiguous()
        s["weights"] = torch.softmax(top.values, 1).contiguous()
        if c["op"] == "sort" and c["direction"] == "forward":
            s["X"], s["Xs"] = normal(T, d), empty(R, d)
            return s
        s["pos"] = _plan(c, ids)[4]                 # a plan that an earlier call made
        if c["op"] == "sort":
            s["dXs"], s["dX"] = normal(R, d), empty(T, d)
        elif c["direction"] == "forward":
            s["O"], s["Y"] = normal(R, d), empty(T, d)
        else:
            s["O"], s["dY"] = normal(R, d), normal(T, d)
            s["dO"], s["dweights"] = empty(R, d), empty(T, k, dtype=torch.float32)
        return s
    size = torch.exp(0.5 * torch.randn(T, 1, generator=g, device="cuda"))          # tokens of different length
    gain = lambda: 1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")          # noqa: E731
    rstd = lambda x: torch.rsqrt(x.float().square().mean(1) + EPS)                 # noqa: E731
    if c["op"] == "norm":
        s["X"], s["w"] = normal(T, d).mul_(size.to(dt)), gain()
        if c["direction"] == "forward":
            s["N"], s["rstd"] = empty(T, d), empty(T, dtype=torch.float32)
        else:
            s["rstd"], s["dN"], s["dres"] = rstd(s["X"]), normal(T, d), normal(T, d)
            s["dX"], s["dw"] = empty(T, d), empty(d, dtype=torch.float32)
        return s
    s["Y"] = normal(T, d).mul_((0.3 * size).to(dt))
    s["w_post"] = gain()
    s["gate"] = torch.sigmoid(torch.randn(T, generator=g, device="cuda")) if c["gate"] else None
    s["w_next"] = gain() if c["next"] else None
    if c["direction"] == "forward":
        s["X"], s["Xo"] = normal(T, d), empty(T, d)
        s["N"] = empty(T, d) if c["next"] else None
        s["rstd_y"] = empty(T, dtype=torch.float32) if c["post"] else None
        s["rstd_o"] = empty(T, dtype=torch.float32) if c["next"] else None
    else:
        s["Xo"] = normal(T, d).mul_(size.to(dt)) if c["next"] else None
        s["dXo"], s["dN"] = normal(T, d), normal(T, d) if c["next"] else None
        s["rstd_y"] = rstd(s["Y"]) if c["post"] else None
        s["rstd_o"] = rstd(s["Xo"]) if c["next"] else None
        s["dX"], s["dY"], s["dw_post"] = empty(T, d), empty(T, d), empty(d, dtype=torch.float32)
        s["dgate"] = empty(T, dtype=torch.float32) if c["gate"] else None
        s["dw_next"] = empty(d, dtype=torch.float32) if c["next"] else None
    return s


# ---- the plain forms ----------------------------------------------------------------------------


def _plan(c, ids):
    """counts [E], offsets [E + 1], totals [4], row_token [rows], pos [T, k] of a choice."""
    T, k, E, R = c["T"], c["k"], c["E"], _n_rows(c)
    flat = ids.reshape(-1)
    key = torch.where((flat >= 0) & (flat < E), flat, E)
    key, order = torch.sort(key, stable=True)
    first = torch.searchsorted(key, torch.arange(E + 1, device=ids.device, dtype=torch.int32))
    found = first[1:] - first[:-1]
    if c["capacity"]:
        stride = (c["capacity"] + 127) // 128 * 128
        counts = found.clamp(max=c["capacity"])
        offsets = torch.arange(E + 1, device=ids.device) * stride
    else:
        counts = found
        ends = torch.cumsum((counts + c["align"] - 1) // c["align"] * c["align"], 0)
        offsets = torch.cat([torch.zeros(1, dtype=ends.dtype, device=ids.device), ends])
    rank = torch.arange(T * k, device=ids.device) - first[key]
    kept = (key < E) & (rank < torch.cat([counts, counts.new_zeros(1)])[key])
    row = torch.where(kept, offsets[key] + rank, -1)
    pos = torch.empty_like(row).scatter_(0, order, row)
    row_token = torch.full((R + 1,), -1, device=ids.device, dtype=torch.int64)
    row_token[torch.where(kept, row, R)] = order // k
    kept_n, all_n = counts.sum(), found.sum()
    totals = torch.stack([kept_n, all_n - kept_n, T * k - all_n, torch.zeros_like(all_n)])
    i32 = torch.int32
    return counts.to(i32), offsets.to(i32), totals.to(i32), row_token[:R].to(i32), pos.to(i32).reshape(T, k)


def _picked(rows, pos):
    """rows[pos] in fp32 [T, k, d], zeros where there is no row."""
    return torch.where((pos >= 0)[..., None], rows[pos.clamp(min=0).long()].float(), 0.0)


def _normed_bwd(g, xhat, rstd):
    return rstd[:, None] * (g - xhat * (g * xhat).mean(1, keepdim=True))


def _plain(s):
    c, dt = s["c"], _dtype(s["c"])
    op = (c["op"], c["direction"])
    if op == ("sort", "forward"):
        counts, offsets, totals, row_token, pos = _plan(c, s["ids"])
        Xs = torch.where((row_token >= 0)[:, None], s["X"][row_token.clamp(min=0).long()], 0.0)
        return {"counts": counts, "offsets": offsets, "totals": totals, "row_token": row_token, "pos": pos, "Xs": Xs}
    if op == ("sort", "backward"):
        return {"dX": _picked(s["dXs"], s["pos"]).sum(1).to(dt)}
    if op == ("unsort", "forward"):
        return {"Y": (s["weights"][..., None] * _picked(s["O"], s["pos"])).sum(1).to(dt)}
    if op == ("unsort", "backward"):
        pos, dY = s["pos"], s["dY"].float()
        dw = (dY[:, None] * _picked(s["O"], pos)).sum(2)
        at = torch.where(pos >= 0, pos, _n_rows(c)).long()
        dO = torch.zeros(_n_rows(c) + 1, c["d"], dtype=dt, device=pos.device)
        dO[at] = (s["weights"][..., None] * dY[:, None]).to(dt)
        return {"dO": dO[:-1], "dweights": dw}
    if op == ("norm", "forward"):
        x = s["X"].float()
        rstd = torch.rsqrt(x.square().mean(1) + EPS)
        return {"N": (x * rstd[:, None] * s["w"]).to(dt), "rstd": rstd}
    if op == ("norm", "backward"):
        dN, xhat = s["dN"].float(), s["X"].float() * s["rstd"][:, None]
        dX = s["dres"].float() + _normed_bwd(dN * s["w"], xhat, s["rstd"])
        return {"dX": dX.to(dt), "dw": (dN * xhat).sum(0)}
    if op == ("join", "forward"):
        y, out = s["Y"].float(), {}
        if c["post"]:
            out["rstd_y"] = torch.rsqrt(y.square().mean(1) + EPS)
            y = y * out["rstd_y"][:, None]
        y = BRANCH_SCALE * y * s["w_post"]
        xo = RES_SCALE * s["X"].float() + (y * s["gate"][:, None] if c["gate"] else y)
        out["Xo"] = xo.to(dt)
        if c["next"]:
            out["rstd_o"] = torch.rsqrt(xo.square().mean(1) + EPS)
            out["N"] = (xo * out["rstd_o"][:, None] * s["w_next"]).to(dt)
        return out
    out, G = {}, s["dXo"].float()
    if c["next"]:
        dN, xhat = s["dN"].float(), s["Xo"].float() * s["rstd_o"][:, None]
        out["dw_next"] = (dN * xhat).sum(0)
        G = G + _normed_bwd(dN * s["w_next"], xhat, s["rstd_o"])
    out["dX"] = (RES_SCALE * G).to(dt)
    y = s["Y"].float()
    yhat = y * s["rstd_y"][:, None] if c["post"] else y
    G = BRANCH_SCALE * G
    if c["gate"]:
        out["dgate"] = (G * yhat * s["w_post"]).sum(1)
        G = G * s["gate"][:, None]
    out["dw_post"] = (G * yhat).sum(0)
    u = G * s["w_post"]
    out["dY"] = (_normed_bwd(u, yhat, s["rstd_y"]) if c["post"] else u).to(dt)
    return out


# ---- the framework's operators --------------------------------------------------------------------


def _handle(s):
    """The binding, the call's configuration and the buffers that a program keeps beside its tensors."""
    if "handle" not in s:
        from paper_2406_00023_b200 import etr
        c = s["c"]
        dtype = etr.BF16 if c["dtype"] == "bf16" else etr.F32
        if c["op"] in ("sort", "unsort"):
            cfg = etr.make_sort_config(T=c["T"], k=c["k"], E=c["E"], d=c["d"], dtype=dtype, align=c["align"], capacity=c["capacity"])
            buf = etr.SortBuffers(cfg)
            if "pos" in s:
                etr.sort(cfg, s["ids"], buf)
        else:
            cfg = etr.make_norm_config(T=c["T"], d=c["d"], dtype=dtype, eps=EPS, res_scale=RES_SCALE, branch_scale=BRANCH_SCALE,
                                       post_norm=c.get("post", True))
            buf = torch.empty(etr.norm_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        s["handle"] = etr, cfg, buf
    return s["handle"]


def _framework(s):
    etr, cfg, buf = _handle(s)
    c = s["c"]
    op = (c["op"], c["direction"])
    if op == ("sort", "forward"):
        etr.sort(cfg, s["ids"], buf)
        etr.sort_rows(cfg, s["X"], buf, s["Xs"])
        return {"counts": buf.counts, "offsets": buf.offsets, "totals": buf.totals, "row_token": buf.row_token, "pos": buf.pos, "Xs": s["Xs"]}
    if op == ("sort", "backward"):
        etr.sort_rows_bwd(cfg, s["dXs"], buf, s["dX"])
        return {"dX": s["dX"]}
    if op == ("unsort", "forward"):
        etr.unsort_rows(cfg, s["O"], s["weights"], buf, s["Y"])
        return {"Y": s["Y"]}
    if op == ("unsort", "backward"):
        etr.unsort_rows_bwd(cfg, s["dY"], s["O"], s["weights"], buf, s["dO"], s["dweights"])
        return {"dO": s["dO"], "dweights": s["dweights"]}
    if op == ("norm", "forward"):
        etr.prenorm(cfg, s["X"], s["w"], s["N"], s["rstd"])
        return {"N": s["N"], "rstd": s["rstd"]}
    if op == ("norm", "backward"):
        etr.prenorm_bwd(cfg, s["dN"], s["X"], s["w"], s["rstd"], s["dres"], s["dX"], s["dw"], buf)
        return {"dX": s["dX"], "dw": s["dw"]}
    if op == ("join", "forward"):
        etr.join(cfg, s["X"], s["Y"], s["w_post"], s["gate"], s["w_next"], s["Xo"], s["N"], s["rstd_y"], s["rstd_o"])
        names = ("Xo", "N", "rstd_y", "rstd_o")
    else:
        etr.join_bwd(cfg, s["dXo"], s["dN"], s["Y"], s["Xo"], s["w_post"], s["gate"], s["w_next"], s["rstd_y"], s["rstd_o"],
                     s["dX"], s["dY"], s["dw_post"], s["dgate"], s["dw_next"], buf)
        names = ("dX", "dY", "dw_post", "dgate", "dw_next")
    return {n: s[n] for n in names if s[n] is not None}


def run(state):
    return _framework(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------


def work(case):
    c = case
    row = c["d"] * (2 if c["dtype"] == "bf16" else 4)
    T, d = c["T"], c["d"]
    op = (c["op"], c["direction"])
    if c["op"] in ("sort", "unsort"):
        pairs = T * c["k"]
        if c["capacity"]:
            pairs = min(pairs, c["E"] * c["capacity"])
        pairs = max(1, round(pairs * (1.0 - c["lost"])))
        if op == ("sort", "forward"):
            return {"bytes": (T + pairs) * row + 4 * (2 * T * c["k"] + _n_rows(c) + 2 * c["E"]), "flops": 0}
        if op == ("sort", "backward"):
            return {"bytes": (T + pairs) * row + 4 * T * c["k"], "flops": pairs * d}
        if op == ("unsort", "forward"):
            return {"bytes": (T + pairs) * row + 8 * T * c["k"], "flops": 2 * pairs * d}
        return {"bytes": (T + 2 * pairs) * row + 12 * T * c["k"], "flops": 3 * pairs * d}
    if op == ("norm", "forward"):
        return {"bytes": 2 * T * row + 4 * T + 4 * d, "flops": 4 * T * d}
    if op == ("norm", "backward"):
        return {"bytes": 4 * T * row + 4 * T + 8 * d, "flops": 10 * T * d}
    tensors = 4 if c["next"] else 3
    if op == ("join", "forward"):
        return {"bytes": tensors * T * row + 12 * T + 8 * d, "flops": 12 * T * d}
    return {"bytes": (tensors + 2 if c["next"] else 4) * T * row + 16 * T + 16 * d, "flops": 24 * T * d}


# ---- the definitions in 64 bits --------------------------------------------------------------------


def exact(case, seed):
    c, s = case, prepare(case, seed)
    f64 = lambda n: s[n].double()              # noqa: E731
    T, d = c["T"], c["d"]
    op = (c["op"], c["direction"])
    if c["op"] in ("sort", "unsort"):
        E, k, R = c["E"], c["k"], _n_rows(c)
        flat = s["ids"].reshape(-1).long()
        hit = flat[:, None] == torch.arange(E, device=flat.device)                  # [T k, E]
        seen = torch.cumsum(hit.to(torch.int32), 0)
        n = seen[-1].long()
        rank = ((seen - 1) * hit).sum(1)
        limit = c["capacity"] or T * k
        counts = torch.minimum(n, torch.full_like(n, limit))
        if c["capacity"]:
            starts = torch.arange(E + 1, device=flat.device) * (-(-c["capacity"] // 128) * 128)
        else:
            starts = torch.zeros(E + 1, dtype=torch.int64, device=flat.device)
            starts[1:] = torch.cumsum(-(-counts // c["align"]) * c["align"], 0)
        live = hit.any(1) & (rank < limit)
        row = starts[flat.clamp(min=0)] + rank
        pair = torch.nonzero(live).flatten()
        at, token = row[pair], pair // k
        if op == ("sort", "forward"):
            row_token = torch.full((R,), -1, dtype=torch.int32, device=flat.device)
            row_token[at] = token.to(torch.int32)
            pos = torch.where(live, row, -1).to(torch.int32).reshape(T, k)
            totals = torch.tensor([int(counts.sum()), int((n - counts).sum()), int(T * k - n.sum()), 0], dtype=torch.int32)
            Xs = torch.zeros(R, d, dtype=torch.float64, device=flat.device)
            Xs[at] = f64("X")[token]
            return {"counts": counts.to(torch.int32), "offsets": starts.to(torch.int32), "totals": totals, "row_token": row_token, "pos": pos, "Xs": Xs}
        out = torch.zeros(T, d, dtype=torch.float64, device=flat.device)
        w = f64("weights").reshape(-1)[pair]
        if op == ("sort", "backward"):
            return {"dX": out.index_add_(0, token, f64("dXs")[at])}
        if op == ("unsort", "forward"):
            return {"Y": out.index_add_(0, token, w[:, None] * f64("O")[at])}
        dY = f64("dY")[token]
        dw = torch.zeros(T * k, dtype=torch.float64, device=flat.device)
        dw[pair] = torch.linalg.vecdot(dY, f64("O")[at])
        dO = torch.zeros(R, d, dtype=torch.float64, device=flat.device)
        dO[at] = w[:, None] * dY
        return {"dO": dO, "dweights": dw.reshape(T, k)}
    if op == ("norm", "forward"):
        x = f64("X")
        inv = (x.pow(2).sum(1) / d + EPS).pow(-0.5)
        return {"N": inv[:, None] * x * f64("w"), "rstd": inv}
    if op == ("norm", "backward"):
        inv, x = f64("rstd")[:, None], f64("X")
        g = f64("dN") * f64("w")
        dX = f64("dres") + inv * g - inv ** 3 * x * torch.linalg.vecdot(g, x)[:, None] / d
        return {"dX": dX, "dw": torch.einsum("td,td,t->d", f64("dN"), x, inv[:, 0])}
    gate = f64("gate")[:, None] if c["gate"] else torch.ones(T, 1, dtype=torch.float64, device=s["Y"].device)
    y, wp = f64("Y"), f64("w_post")
    if op == ("join", "forward"):
        inv = (y.pow(2).sum(1) / d + EPS).pow(-0.5) if c["post"] else None
        branch = gate * wp * (y * inv[:, None] if c["post"] else y)
        xo = RES_SCALE * f64("X") + BRANCH_SCALE * branch
        out = {"Xo": xo}
        if c["post"]:
            out["rstd_y"] = inv
        if c["next"]:
            out["rstd_o"] = (xo.pow(2).sum(1) / d + EPS).pow(-0.5)
            out["N"] = xo * out["rstd_o"][:, None] * f64("w_next")
        return out
    out, G = {}, f64("dXo")
    if c["next"]:
        dN, xo, inv = f64("dN"), f64("Xo"), f64("rstd_o")[:, None]
        g = dN * f64("w_next")
        out["dw_next"] = torch.einsum("td,td,t->d", dN, xo, inv[:, 0])
        G = G + inv * g - inv ** 3 * xo * torch.linalg.vecdot(g, xo)[:, None] / d
    out["dX"] = RES_SCALE * G
    inv = f64("rstd_y")[:, None] if c["post"] else torch.ones_like(gate)
    if c["gate"]:
        out["dgate"] = BRANCH_SCALE * inv[:, 0] * torch.linalg.vecdot(G * wp, y)
    out["dw_post"] = BRANCH_SCALE * torch.einsum("td,td,t->d", G, y, (inv * gate)[:, 0])
    u = BRANCH_SCALE * gate * G * wp
    out["dY"] = inv * u - (inv ** 3 * y * torch.linalg.vecdot(u, y)[:, None] / d if c["post"] else 0.0)
    return out
