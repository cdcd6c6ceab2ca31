"""The norm before a block and the join behind it, on the GPU, against their 64-bit definitions (tests/rows_reference.py has the
bounds)."""
import itertools

import pytest
import torch

from paper_2406_00023_b200 import etr
from tests import rows_reference as rr

pytestmark = pytest.mark.gpu
DT = {torch.bfloat16: etr.BF16, torch.float32: etr.F32}
TYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
EPS, A, B = 1e-6, 0.875, 0.5
SIZES = [(1, 8), (3, 64), (2, 256), (17, 264), (9, 512), (5, 520), (33, 768), (64, 1024), (31, 1088), (7, 2048), (300, 2056), (13, 4096),
         (5, 8192), (3, 8200), (4, 16384), (2000, 16), (1531, 768),
         (2500, 1088), (1300, 4096), (700, 8192), (300, 12288)]


def tensors(T, d, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = lambda s=1.0: (torch.randn(T, d, generator=g, device="cuda") * torch.exp(torch.randn(T, 1, generator=g, device="cuda")) * s).to(dtype)   # noqa: E731
    gain = lambda: 1 + 0.3 * torch.randn(d, generator=g, device="cuda")                                # noqa: E731
    return rows, gain, torch.rand(T, generator=g, device="cuda")


def nans(*shape, dtype=torch.float32):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def workspace(cfg):
    return nans(etr.norm_workspace_bytes(cfg) // 4)


@TYPES
@pytest.mark.parametrize("T, d", SIZES)
@pytest.mark.parametrize("gain", [True, False])
def test_prenorm(T, d, dtype, gain):
    cfg = etr.make_norm_config(T=T, d=d, dtype=DT[dtype], eps=EPS)
    rows, gains, _ = tensors(T, d, dtype, T + d)
    X, w, dN, dres = rows(), gains() if gain else None, rows(), rows()
    if T > 2:
        X[1] = 0                                           # a row of zeros: 1 / sqrt(eps)
    N, r = nans(T, d, dtype=dtype), nans(T)
    etr.prenorm(cfg, X, w, N, r)
    (ref, bound), (r_ref, r_bound) = rr.prenorm(X, w, EPS, dtype)
    rr.assert_within(N, ref, bound, "N")
    rr.assert_within(r, r_ref, r_bound, "rstd")
    N2 = nans(T, d, dtype=dtype)
    etr.prenorm(cfg, X, w, N2)
    assert torch.equal(N, N2)
    for res, want_dw in ((dres, True), (None, True), (dres, False)):
        dX, dw = nans(T, d, dtype=dtype), nans(d) if want_dw else None
        etr.prenorm_bwd(cfg, dN, X, w, r, res, dX, dw, workspace(cfg) if want_dw else None)
        x, g = rr.prenorm_bwd(dN, X, w, r, res, dtype)
        rr.assert_within(dX, *x, "dX")
        if want_dw:
            rr.assert_within(dw, *g, "dw")


OPTIONS = list(itertools.product([True, False], repeat=4))


@TYPES
@pytest.mark.parametrize("T, d", SIZES)
@pytest.mark.parametrize("post, gated, gain, follow", OPTIONS[::3] + [OPTIONS[-1]])
def test_join(T, d, dtype, post, gated, gain, follow):
    cfg = etr.make_norm_config(T=T, d=d, dtype=DT[dtype], eps=EPS, res_scale=A, branch_scale=B, post_norm=post)
    rows, gains, gate = tensors(T, d, dtype, T + 3 * d)
    X, Y, dXo, dN = rows(), rows(0.3), rows(), rows()
    wp, wn = (gains(), gains()) if gain else (None, None)
    gate = gate if gated else None
    if T > 2:
        Y[0] = 0
    Xo, N, ry, ro = nans(T, d, dtype=dtype), nans(T, d, dtype=dtype) if follow else None, nans(T), nans(T)
    etr.join(cfg, X, Y, wp, gate, wn, Xo, N, ry, ro)
    ref = rr.join(X, Y, wp, gate, wn, EPS, A, B, post, dtype)
    rr.assert_within(Xo, *ref["Xo"], "Xo")
    if post:
        rr.assert_within(ry, *ref["rstd_y"], "rstd_y")
    if follow:
        rr.assert_within(N, *ref["N"], "N")
        rr.assert_within(ro, *ref["rstd_o"], "rstd_o")
    for use_dxo, wanted in ((True, True), (False, True), (True, False)):
        if not use_dxo and not follow:
            continue
        dX, dY = nans(T, d, dtype=dtype), nans(T, d, dtype=dtype)
        dwp, dg, dwn = (nans(d), nans(T), nans(d) if follow else None) if wanted else (None, None, None)
        etr.join_bwd(cfg, dXo if use_dxo else None, dN if follow else None, Y, Xo if follow else None, wp, gate, wn, ry if post else None,
                     ro if follow else None, dX, dY, dwp, dg, dwn, workspace(cfg) if wanted else None)
        ref = rr.join_bwd(dXo if use_dxo else None, dN if follow else None, Y, Xo, wp, gate, wn, ry, ro, A, B, post, dtype)
        for name, got in (("dX", dX), ("dY", dY), ("dw_post", dwp), ("dgate", dg), ("dw_next", dwn)):
            if got is not None:
                rr.assert_within(got, *ref[name], name)


@TYPES
def test_gains_gradients_over_many_rows(dtype):
    """More rows than the backward kernels have blocks: every block walks several."""
    for T, d in ((5000, 256), (3000, 1088), (1300, 4096)):
        cfg = etr.make_norm_config(T=T, d=d, dtype=DT[dtype], eps=EPS, res_scale=A, branch_scale=B, post_norm=True)
        rows, gains, gate = tensors(T, d, dtype, T)
        Y, Xo, dXo, dN, wp, wn = rows(), rows(), rows(), rows(), gains(), gains()
        ry, ro = (rr.prenorm(x, None, EPS, dtype)[1][0].float() for x in (Y, Xo))
        out = dict(dX=nans(T, d, dtype=dtype), dY=nans(T, d, dtype=dtype), dw_post=nans(d), dgate=nans(T), dw_next=nans(d))
        etr.join_bwd(cfg, dXo, dN, Y, Xo, wp, gate, wn, ry, ro, *out.values(), workspace(cfg))
        ref = rr.join_bwd(dXo, dN, Y, Xo, wp, gate, wn, ry, ro, A, B, True, dtype)
        for name in out:
            rr.assert_within(out[name], *ref[name], name)
        again = {n: torch.empty_like(t) for n, t in out.items()}
        etr.join_bwd(cfg, dXo, dN, Y, Xo, wp, gate, wn, ry, ro, *again.values(), workspace(cfg))
        assert all(torch.equal(out[n], again[n]) for n in out)                     # the sums' order is fixed
        dX, dw = nans(T, d, dtype=dtype), nans(d)
        etr.prenorm_bwd(cfg, dN, Xo, wn, ro, None, dX, dw, workspace(cfg))
        x, g = rr.prenorm_bwd(dN, Xo, wn, ro, None, dtype)
        rr.assert_within(dX, *x, "dX")
        rr.assert_within(dw, *g, "dw")


@pytest.mark.parametrize("d", [256, 1088, 4096])
def test_in_place_residual(d):
    """Xo may be X, and dX may be dXo or dres: the bits of the call with separate outputs."""
    T, dtype = 400, torch.bfloat16
    cfg = etr.make_norm_config(T=T, d=d, dtype=etr.BF16, eps=EPS, res_scale=A, branch_scale=B, post_norm=True)
    rows, gains, gate = tensors(T, d, dtype, d)
    X, Y, dXo, dN, wp, wn = rows(), rows(), rows(), rows(), gains(), gains()
    Xo, N, N2, ry, ro = torch.empty_like(X), torch.empty_like(X), torch.empty_like(X), nans(T), nans(T)
    etr.join(cfg, X, Y, wp, gate, wn, Xo, N, ry, ro)
    stream = X.clone()
    etr.join(cfg, stream, Y, wp, gate, wn, stream, N2, ry, ro)
    assert torch.equal(stream, Xo) and torch.equal(N, N2)
    dX, dY, dY2, ws = torch.empty_like(X), torch.empty_like(X), torch.empty_like(X), workspace(cfg)
    etr.join_bwd(cfg, dXo, dN, Y, Xo, wp, gate, wn, ry, ro, dX, dY, nans(d), nans(T), nans(d), ws)
    stream = dXo.clone()
    etr.join_bwd(cfg, stream, dN, Y, Xo, wp, gate, wn, ry, ro, stream, dY2, nans(d), nans(T), nans(d), ws)
    assert torch.equal(stream, dX) and torch.equal(dY, dY2)
    etr.prenorm_bwd(cfg, dN, X, wn, ro, dXo, dX, nans(d), ws)
    stream = dXo.clone()
    etr.prenorm_bwd(cfg, dN, X, wn, ro, stream, stream, nans(d), ws)
    assert torch.equal(stream, dX)


def test_empty_batches():
    cfg = etr.make_norm_config(T=0, d=64, dtype=etr.BF16, post_norm=True)
    e, r, dw, dwn, ws = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(0, device="cuda"), nans(64), nans(64), workspace(cfg)
    etr.prenorm(cfg, e, None, e.clone(), r)
    etr.join(cfg, e, e, None, None, None, e.clone(), None)
    etr.prenorm_bwd(cfg, e, e, None, r, None, e.clone(), dw, ws)
    assert bool((dw == 0).all())
    dw.fill_(float("nan"))
    etr.join_bwd(cfg, e, e, e, e, None, None, None, r, r, e.clone(), e.clone(), dw, None, dwn, ws)
    assert bool((dw == 0).all()) and bool((dwn == 0).all())


def test_special_values_stay_in_their_row():
    T, d = 20, 1088
    cfg = etr.make_norm_config(T=T, d=d, dtype=etr.BF16, eps=EPS, post_norm=True)
    rows, gains, gate = tensors(T, d, torch.bfloat16, 4)
    X, Y, w = rows(), rows(), gains()
    clean, N, got, N2 = (torch.empty_like(X) for _ in range(4))
    etr.join(cfg, X, Y, w, gate, w, clean, N, None, None)
    X[3, 5], Y[7, 9], gate[11] = float("nan"), float("inf"), float("nan")
    etr.join(cfg, X, Y, w, gate, w, got, N2, None, None)
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[[3, 7, 11]] = False
    assert torch.equal(got[keep], clean[keep]) and torch.equal(N2[keep], N[keep])
    assert bool(N2[3].isnan().all()) and bool(got[11].isnan().all())


def test_small_values_keep_eps_in_charge():
    """Rows far below sqrt(eps) and rows whose squares underflow."""
    for dtype in (torch.bfloat16, torch.float32):
        X = (torch.randn(6, 520, device="cuda") * torch.tensor([1e-3, 1e-5, 1e-12, 1e-25, 1e-30, 1e10], device="cuda")[:, None]).to(dtype)
        cfg = etr.make_norm_config(T=6, d=520, dtype=DT[dtype], eps=EPS)
        N, r = nans(6, 520, dtype=dtype), nans(6)
        etr.prenorm(cfg, X, None, N, r)
        (ref, bound), (r_ref, r_bound) = rr.prenorm(X, None, EPS, dtype)
        rr.assert_within(N, ref, bound, "N")
        rr.assert_within(r, r_ref, r_bound, "rstd")


@TYPES
def test_values_up_to_the_documented_size(dtype):
    """1e17 in the widest rows: the sum of the squares is half of what fp32 holds."""
    T, d = 5, 16384
    X, dN = ((torch.rand(T, d, device="cuda") * 2 - 1).mul_(9.9e16).to(dtype) for _ in range(2))
    X[0] = 9.9e16
    cfg = etr.make_norm_config(T=T, d=d, dtype=DT[dtype], eps=EPS)
    N, r, dX, dw = nans(T, d, dtype=dtype), nans(T), nans(T, d, dtype=dtype), nans(d)
    etr.prenorm(cfg, X, None, N, r)
    (ref, bound), (r_ref, r_bound) = rr.prenorm(X, None, EPS, dtype)
    rr.assert_within(N, ref, bound, "N")
    rr.assert_within(r, r_ref, r_bound, "rstd")
    etr.prenorm_bwd(cfg, dN, X, None, r, None, dX, dw, workspace(cfg))
    x, g = rr.prenorm_bwd(dN, X, None, r, None, dtype)
    rr.assert_within(dX, *x, "dX")
    rr.assert_within(dw, *g, "dw")


def test_captured_calls_and_another_stream():
    T, d = 300, 1024
    cfg = etr.make_norm_config(T=T, d=d, dtype=etr.BF16, eps=EPS, res_scale=A, branch_scale=B, post_norm=True)
    rows, gains, gate = tensors(T, d, torch.bfloat16, 8)
    X, Y, dXo, dN, wp, wn = rows(), rows(), rows(), rows(), gains(), gains()
    outs = [torch.empty_like(X) for _ in range(4)] + [nans(T), nans(T), nans(T), nans(d), nans(d)]
    ws = workspace(cfg)

    def calls():
        Xo, N, dX, dY, ry, ro, dg, dwp, dwn = outs
        etr.join(cfg, X, Y, wp, gate, wn, Xo, N, ry, ro)
        etr.join_bwd(cfg, dXo, dN, Y, Xo, wp, gate, wn, ry, ro, dX, dY, dwp, dg, dwn, ws)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    X.copy_(rows())
    Y.copy_(rows())
    graph.replay()
    torch.cuda.synchronize()
    replayed = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        calls()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, replayed))
    rr.assert_within(outs[0], *rr.join(X, Y, wp, gate, wn, EPS, A, B, True, torch.bfloat16)["Xo"], "Xo")


def test_rows_beyond_32_bit_offsets():
    T, d = 140000, 16384
    cfg = etr.make_norm_config(T=T, d=d, dtype=etr.BF16, eps=EPS)
    X = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    X.copy_((1 + torch.arange(T, device="cuda") % 7).bfloat16()[:, None].expand(T, d))
    N, r = torch.empty_like(X), nans(T)
    etr.prenorm(cfg, X, None, N, r)
    assert bool((N == 1).all())
    dw, ws = nans(d), workspace(cfg)
    dX = torch.empty_like(X)
    etr.prenorm_bwd(cfg, N, X, None, r, X, dX, dw, ws)             # N and X are parallel: the norm's part of dX is nothing
    assert bool(((dX.float() - X.float()).abs() <= 0.01).all())
    assert bool(((dw - T).abs() <= T * 1e-4).all())


def test_calls_are_refused_before_a_launch():
    cfg = etr.make_norm_config(T=10, d=64, dtype=etr.BF16)
    X, N = torch.zeros(10, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(10, 64, dtype=torch.bfloat16, device="cuda")
    n0 = etr.launch_count()
    for bad, code in ((X.float(), etr.ERR_ARG), (X[:9], etr.ERR_SHAPE), (X.cpu(), etr.ERR_ARG), (X.t(), etr.ERR_SHAPE),
                      (torch.zeros(641, dtype=torch.bfloat16, device="cuda")[1:], etr.ERR_ALIGN)):
        with pytest.raises(etr.EtrError) as e:
            etr.prenorm(cfg, bad, None, N)
        assert e.value.code == code
    w = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(etr.EtrError) as e:
        etr.prenorm(cfg, X, w, N)                                  # gains are fp32
    assert e.value.code == etr.ERR_ARG
    with pytest.raises(etr.EtrError) as e:
        etr.prenorm_bwd(cfg, N, X, None, torch.zeros(10, device="cuda"), None, X.clone(), torch.zeros(64, device="cuda"), torch.zeros(4, device="cuda"))
    assert e.value.code == etr.ERR_WORKSPACE
    assert etr.launch_count() == n0
