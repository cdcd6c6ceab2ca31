"""Definitions in 64 bits of the operators between the residual stream and the experts (sort, unsort, prenorm, join and their
gradients), with bounds of what 32-bit sums and one rounding per stored value may add.

Bounds: u = 2^-24 is the largest relative error of one fp32 operation; a sum of n fp32 terms, in any order, is off by at most
n u times the sum of the terms' sizes; storing a value in a type rounds it by at most eps / 2 of its size.
"""
from __future__ import annotations

import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def assert_within(got, ref, bound, what):
    got = got.detach().double().to(ref.device)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    bad = ~((got - ref).abs() <= bound + 1e-37)
    assert not bool(bad.any()), (what, int(bad.sum()), float((got - ref).abs()[bad].max()), float((bound + 0 * ref)[bad].max()))


# ---- sort -------------------------------------------------------------------------------------


def plan(ids, E, align, capacity, n_rows):
    """counts, offsets, totals, row_token, pos as lists of int, pair by pair."""
    T, k = ids.shape
    ids = ids.cpu().tolist()
    per = [[] for _ in range(E)]
    none = 0
    for t in range(T):
        for j in range(k):
            if 0 <= ids[t][j] < E:
                per[ids[t][j]].append((t, j))
            else:
                none += 1
    kept = [p[:capacity] if capacity else p for p in per]
    stride = (capacity + 127) // 128 * 128
    offsets = [0]
    for p in kept:
        offsets.append(offsets[-1] + (stride if capacity else (len(p) + align - 1) // align * align))
    row_token, pos = [-1] * n_rows, [[-1] * k for _ in range(T)]
    for e, p in enumerate(kept):
        for i, (t, j) in enumerate(p):
            row_token[offsets[e] + i] = t
            pos[t][j] = offsets[e] + i
    dropped = sum(len(p) for p in per) - sum(len(p) for p in kept)
    return [len(p) for p in kept], offsets, [sum(len(p) for p in kept), dropped, none, 0], row_token, pos


def unsort(rows, w, pos, dtype):
    """Y and its bound; w None: ones."""
    T, k = pos.shape
    picked = torch.where((pos >= 0)[..., None], rows.double()[pos.clamp(min=0).long()], 0.0)
    f = torch.where(pos >= 0, w.double(), 0.0) if w is not None else (pos >= 0).double()
    terms = f[..., None] * picked
    ref, size = terms.sum(1), terms.abs().sum(1)
    err = (k + 1) * U * size
    return ref, err + half_step(dtype) * (ref.abs() + err)


def unsort_bwd(dY, rows, w, pos, n_rows, dtype):
    """(dO with NaN in rows of no pair, its bound), (dweights, its bound)."""
    T, k = pos.shape
    d = dY.shape[1]
    ok = pos >= 0
    picked = torch.where(ok[..., None], rows.double()[pos.clamp(min=0).long()], 0.0)
    terms = dY.double()[:, None] * picked
    dw, dw_err = terms.sum(2), (d + 1) * U * terms.abs().sum(2)
    dO = torch.full((n_rows, d), float("nan"), dtype=torch.float64, device=dY.device)
    pair = (torch.where(ok, w.double(), 0.0)[..., None] * dY.double()[:, None])
    dO[pos[ok].long()] = pair[ok]
    return (dO, dO.abs() * (U + half_step(dtype) * (1 + U))), (dw, dw_err)


# ---- norms ------------------------------------------------------------------------------------


def _rstd(x, err, eps):
    """r(x) in 64 bits and the relative error of its fp32 form, x being off by err: the sum of d squares (d + 1 roundings),
    the quotient, the added eps and the reciprocal root (2 ulp: 4 u)."""
    d = x.shape[1]
    r = (x.pow(2).mean(1) + eps).pow(-0.5)
    off = torch.linalg.vector_norm(err, dim=1) / torch.linalg.vector_norm(x, dim=1).clamp(min=1e-300)
    return r, off + (d + 4) * U / 2 + 4 * U


def prenorm(x, w, eps, dtype):
    x = x.double()
    w = w.double() if w is not None else torch.ones(x.shape[1], dtype=torch.float64, device=x.device)
    r, rel = _rstd(x, torch.zeros_like(x), eps)
    N = x * r[:, None] * w
    return (N, N.abs() * (rel[:, None] + 2 * U + half_step(dtype) * (1 + 1e-3))), (r, r * rel)


def join(X, Y, w_post, gate, w_next, eps, a, b, post, dtype):
    """{name: (value, bound)} of Xo, N, rstd_y, rstd_o."""
    X, Y = X.double(), Y.double()
    one = torch.ones(X.shape[1], dtype=torch.float64, device=X.device)
    wp = w_post.double() if w_post is not None else one
    g = gate.double()[:, None] if gate is not None else torch.ones(X.shape[0], 1, dtype=torch.float64, device=X.device)
    out = {}
    rel_y = torch.zeros_like(g)
    v = Y
    if post:
        r, rel = _rstd(Y, torch.zeros_like(Y), eps)
        out["rstd_y"] = (r, r * rel)
        rel_y, v = rel[:, None], Y * r[:, None]
    branch = b * g * v * wp
    xo = a * X + branch
    # the factors b, r, gate, y, w_post (4 products), a x (1), their sum (1)
    err = branch.abs() * (rel_y + 6 * U) + 3 * U * (a * X).abs()
    # a and b reach the kernel as fp32 numbers: the tests take values that fp32 holds
    out["Xo"] = (xo, err + half_step(dtype) * (xo.abs() + err))
    r, rel = _rstd(xo, err, eps)
    out["rstd_o"] = (r, r * rel)
    wn = w_next.double() if w_next is not None else one
    N = xo * r[:, None] * wn
    err_n = err * r[:, None] * wn.abs() + N.abs() * (rel[:, None] + 3 * U)
    out["N"] = (N, err_n + half_step(dtype) * (N.abs() + err_n))
    return out


def _norm_bwd(g, eg, xh, r):
    """r (g - xh <g, xh> / d) and its bound; g is off by eg, xh by one rounding."""
    d = g.shape[1]
    c = (g * xh).mean(1, keepdim=True)
    ec = ((eg * xh.abs()).sum(1, keepdim=True) + (d + 6) * U * (g * xh).abs().sum(1, keepdim=True)) / d
    return r * (g - xh * c), r * (eg + xh.abs() * ec + 5 * U * (g.abs() + 2 * (xh * c).abs()))


def prenorm_bwd(dN, X, w, rstd, dres, dtype):
    d, T = X.shape[1], X.shape[0]
    dN, r = dN.double(), rstd.double()[:, None]
    xh = X.double() * r
    g = dN * (w.double() if w is not None else 1.0)
    dX, err = _norm_bwd(g, 2 * U * g.abs(), xh, r)
    if dres is not None:
        dX = dX + dres.double()
        err = err + 2 * U * dX.abs()
    dw = dN * xh
    return (dX, err + half_step(dtype) * (dX.abs() + err)), (dw.sum(0), (T + 3) * U * dw.abs().sum(0))


def join_bwd(dXo, dN, Y, Xo, w_post, gate, w_next, rstd_y, rstd_o, a, b, post, dtype):
    """{name: (value, bound)} of dX, dY, dw_post, dgate, dw_next."""
    T, d = Y.shape
    out = {}
    G = dXo.double() if dXo is not None else torch.zeros(T, d, dtype=torch.float64, device=Y.device)
    eG = torch.zeros_like(G)
    if dN is not None:
        r = rstd_o.double()[:, None]
        dn, xh = dN.double(), Xo.double() * r
        g = dn * (w_next.double() if w_next is not None else 1.0)
        part, e = _norm_bwd(g, 2 * U * g.abs(), xh, r)
        G = G + part
        eG = e + 2 * U * G.abs() + U * part.abs()
        out["dw_next"] = ((dn * xh).sum(0), (T + 3) * U * (dn * xh).abs().sum(0))
    dX = a * G
    e = abs(a) * eG + U * dX.abs()
    out["dX"] = (dX, e + half_step(dtype) * (dX.abs() + e))
    wp = w_post.double() if w_post is not None else torch.ones(d, dtype=torch.float64, device=Y.device)
    ga = gate.double()[:, None] if gate is not None else torch.ones(T, 1, dtype=torch.float64, device=Y.device)
    r = rstd_y.double()[:, None] if post else torch.ones_like(ga)
    yh = Y.double() * r
    term = b * G * wp * yh
    e_term = abs(b) * eG * (wp * yh).abs() + 5 * U * term.abs()
    out["dgate"] = (term.sum(1), e_term.sum(1) + (d + 1) * U * term.abs().sum(1))
    pw = b * ga * G * yh
    out["dw_post"] = (pw.sum(0), (abs(b) * ga * eG * yh.abs()).sum(0) + (T + 5) * U * pw.abs().sum(0))
    u = b * ga * wp * G
    eu = (b * ga * wp).abs() * eG + 4 * U * u.abs()
    if post:
        dY, e = _norm_bwd(u, eu, yh, r)
    else:
        dY, e = u, eu + 2 * U * u.abs()
    out["dY"] = (dY, e + half_step(dtype) * (dY.abs() + e))
    return out
