"""The 64-bit definitions that the GPU tests hold the row operators to: gradients against central differences of the forward
forms, and the refusals of the C entry points, none of which need a GPU."""
import ctypes as C

import pytest
import torch

from tests import rows_reference as rr
from paper_2406_00023_b200 import etr

F64 = torch.float64


def differences(f, x, step=1e-5):
    """Gradient of the scalar f by central differences."""
    g = torch.zeros_like(x)
    for i in range(x.numel()):
        keep = float(x.view(-1)[i])
        x.view(-1)[i] = keep + step
        up = float(f())
        x.view(-1)[i] = keep - step
        down = float(f())
        x.view(-1)[i] = keep
        g.view(-1)[i] = (up - down) / (2 * step)
    return g


def close(got, ref):
    assert torch.allclose(got, ref, rtol=1e-6, atol=1e-7), float((got - ref).abs().max())


@pytest.mark.parametrize("gain", [True, False])
def test_prenorm_gradient_is_the_forward_forms_slope(gain):
    g = torch.Generator().manual_seed(1)
    x, dN, dres = (torch.randn(3, 8, generator=g, dtype=F64) for _ in range(3))
    w = torch.randn(8, generator=g, dtype=F64) if gain else None
    f = lambda: (rr.prenorm(x, w, 1e-3, torch.float64)[0][0] * dN).sum() + (x * dres).sum()      # noqa: E731
    r = rr.prenorm(x, w, 1e-3, torch.float64)[1][0]
    (dX, _), (dw, _) = rr.prenorm_bwd(dN, x, w, r, dres, torch.float64)
    close(dX, differences(f, x))
    if gain:
        close(dw, differences(f, w))


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("use_next", [True, False])
@pytest.mark.parametrize("use_dxo", [True, False])
def test_join_gradients_are_the_forward_forms_slopes(post, use_next, use_dxo):
    if not use_next and not use_dxo:
        return
    g = torch.Generator().manual_seed(2)
    T, d, a, b, eps = 3, 8, 0.75, -0.5, 1e-3
    X, Y, dXo, dN = (torch.randn(T, d, generator=g, dtype=F64) for _ in range(4))
    wp, wn = torch.randn(d, generator=g, dtype=F64), torch.randn(d, generator=g, dtype=F64)
    gate = torch.rand(T, generator=g, dtype=F64)
    fwd = lambda: rr.join(X, Y, wp, gate, wn, eps, a, b, post, torch.float64)                       # noqa: E731

    def f():
        o = fwd()
        return (o["Xo"][0] * dXo).sum() * use_dxo + (o["N"][0] * dN).sum() * use_next

    o = fwd()
    grad = rr.join_bwd(dXo if use_dxo else None, dN if use_next else None, Y, o["Xo"][0], wp, gate, wn,
                       o["rstd_y"][0] if post else None, o["rstd_o"][0], a, b, post, torch.float64)
    for name, x in (("dX", X), ("dY", Y), ("dw_post", wp), ("dgate", gate)) + ((("dw_next", wn),) if use_next else ()):
        close(grad[name][0], differences(f, x))


def test_unsort_gradients_are_the_forward_forms_slopes():
    g = torch.Generator().manual_seed(3)
    ids = torch.tensor([[0, 2], [2, 2], [-1, 1], [3, 0]])
    n = 9
    pos = torch.tensor(rr.plan(ids, 3, 1, 0, n)[4])
    O, w, dY = (torch.randn(*s, generator=g, dtype=F64) for s in ((n, 8), (4, 2), (4, 8)))
    f = lambda: (rr.unsort(O, w, pos, F64)[0] * dY).sum()                                          # noqa: E731
    (dO, _), (dw, _) = rr.unsort_bwd(dY, O, w, pos, n, F64)
    close(torch.nan_to_num(dO), differences(f, O))
    close(dw, differences(f, w))
    X = torch.randn(4, 8, generator=g, dtype=F64)
    dXs = torch.randn(n, 8, generator=g, dtype=F64)
    spread = lambda: sum(float((X[t] * dXs[pos[t, j]]).sum()) for t in range(4) for j in range(2) if pos[t, j] >= 0)   # noqa: E731
    close(rr.unsort(dXs, None, pos, F64)[0], differences(spread, X))


def test_plan_by_hand():
    ids = torch.tensor([[1, 0], [1, 5], [0, 1], [-1, 1]])
    assert rr.plan(ids, 2, 1, 0, 8) == ([2, 4], [0, 2, 6], [6, 0, 2, 0], [0, 2, 0, 1, 2, 3, -1, -1], [[2, 0], [3, -1], [1, 4], [-1, 5]])
    assert rr.plan(ids, 2, 4, 0, 14)[1:3] == ([0, 4, 8], [6, 0, 2, 0])
    counts, offsets, totals, _, pos = rr.plan(ids, 2, 128, 3, 256)
    assert (counts, offsets, totals, pos[3]) == ([2, 3], [0, 128, 256], [5, 1, 2, 0], [-1, -1])


# ---- refusals: status codes before any launch (there is no GPU here: a launch would fail with another status) -----


def pointers():
    """The library with plain addresses for arguments."""
    L = etr.lib()
    for name, n in (("etr_sort", 4), ("etr_sort_rows", 5), ("etr_sort_rows_bwd", 5), ("etr_unsort_rows", 6), ("etr_unsort_rows_bwd", 8),
                    ("etr_prenorm", 6), ("etr_prenorm_bwd", 10), ("etr_join", 11), ("etr_join_bwd", 17)):
        getattr(L, name).argtypes = [C.c_void_p] * n
    return L


def sort_cfg(**kw):
    return etr.make_sort_config(**dict(dict(T=4, k=2, E=3, d=16, dtype=etr.BF16), **kw))


@pytest.mark.parametrize("change, code", [
    (dict(), etr.OK), (dict(T=0), etr.OK), (dict(T=-1), etr.ERR_ARG), (dict(k=0), etr.ERR_ARG), (dict(k=33), etr.ERR_SHAPE),
    (dict(k=32), etr.OK), (dict(E=0), etr.ERR_ARG), (dict(E=1024), etr.OK), (dict(E=1025), etr.ERR_SHAPE), (dict(d=12), etr.ERR_SHAPE),
    (dict(d=0), etr.ERR_ARG), (dict(dtype=2), etr.ERR_ARG), (dict(align=0), etr.ERR_ARG), (dict(align=1025), etr.ERR_SHAPE),
    (dict(capacity=-1), etr.ERR_ARG), (dict(capacity=5), etr.ERR_SHAPE), (dict(capacity=5, align=128), etr.OK),
    (dict(T=1 << 30), etr.ERR_SHAPE), (dict(E=1024, capacity=1 << 21, align=128), etr.ERR_SHAPE)])
def test_sort_configurations(change, code):
    cfg = sort_cfg(**change)
    assert etr.sort_validate(cfg) == code
    if code != etr.OK:
        assert etr.sort_n_rows(cfg) == 0
        n = C.c_size_t(0)
        assert etr.lib().etr_sort_plan_bind(C.byref(cfg), None, C.c_size_t(0), None, C.byref(n)) == code
        plan = etr.SortPlan(*[1 << 20] * 6)
        assert pointers().etr_sort(C.addressof(cfg), 1 << 20, C.addressof(plan), None) == code


def test_sort_rows_of_the_buffers():
    assert etr.sort_n_rows(sort_cfg()) == 8
    assert etr.sort_n_rows(sort_cfg(align=16)) == 8 + 3 * 15
    assert etr.sort_n_rows(sort_cfg(T=1, E=100, align=16)) == 2 + 2 * 15
    assert etr.sort_n_rows(sort_cfg(capacity=129, align=128)) == 3 * 256
    assert etr.sort_n_rows(sort_cfg(T=0)) == 0


def test_sort_pointers_are_checked():
    L, cfg, ok = pointers(), sort_cfg(), 1 << 20
    a = C.addressof(cfg)

    def plan(**kw):
        p = etr.SortPlan(*[ok] * 6)
        for n, v in kw.items():
            setattr(p, n, v)
        return p

    for name in ("counts", "offsets", "totals", "row_token", "pos", "scratch"):
        for value, code in ((None, etr.ERR_ARG), (ok + 4, etr.ERR_ALIGN)):
            p = plan(**{name: value})
            q = C.addressof(p)
            assert L.etr_sort(a, ok, q, None) == code
            assert L.etr_sort_rows(a, ok, q, ok, None) == code
            assert L.etr_sort_rows_bwd(a, ok, q, ok, None) == code
            assert L.etr_unsort_rows(a, ok, ok, q, ok, None) == code
            assert L.etr_unsort_rows_bwd(a, ok, ok, ok, q, ok, ok, None) == code
    p = plan()
    q = C.addressof(p)
    for bad, code in ((None, etr.ERR_ARG), (ok + 8, etr.ERR_ALIGN)):
        assert L.etr_sort(a, bad, q, None) == code
        for call, n in ((lambda v: L.etr_sort_rows(a, v[0], q, v[1], None), 2), (lambda v: L.etr_sort_rows_bwd(a, v[0], q, v[1], None), 2),
                        (lambda v: L.etr_unsort_rows(a, v[0], v[1], q, v[2], None), 3),
                        (lambda v: L.etr_unsort_rows_bwd(a, v[0], v[1], v[2], q, v[3], v[4], None), 5)):
            for i in range(n):
                assert call([bad if j == i else ok for j in range(n)]) == code
    assert L.etr_sort(None, ok, q, None) == etr.ERR_ARG and L.etr_sort(a, ok, None, None) == etr.ERR_ARG
    n, out = C.c_size_t(0), etr.SortPlan()
    assert L.etr_sort_plan_bind(a, None, C.c_size_t(0), None, C.byref(n)) == etr.OK and n.value % 256 == 0
    assert L.etr_sort_plan_bind(a, C.c_void_p(ok + 16), n, C.byref(out), None) == etr.ERR_ALIGN
    assert L.etr_sort_plan_bind(a, C.c_void_p(ok), C.c_size_t(n.value - 1), C.byref(out), None) == etr.ERR_WORKSPACE
    assert L.etr_sort_plan_bind(a, C.c_void_p(ok), n, C.byref(out), None) == etr.OK and out.counts == ok


def norm_cfg(**kw):
    return etr.make_norm_config(**dict(dict(T=4, d=16, dtype=etr.BF16, post_norm=True), **kw))


@pytest.mark.parametrize("change, code", [
    (dict(), etr.OK), (dict(T=0), etr.OK), (dict(T=-1), etr.ERR_ARG), (dict(d=0), etr.ERR_ARG), (dict(d=20), etr.ERR_SHAPE),
    (dict(d=16384), etr.OK), (dict(d=16392), etr.ERR_SHAPE), (dict(dtype=7), etr.ERR_ARG), (dict(eps=0.0), etr.ERR_ARG),
    (dict(eps=float("nan")), etr.ERR_ARG), (dict(eps=float("inf")), etr.ERR_ARG), (dict(eps=-1e-6), etr.ERR_ARG),
    (dict(res_scale=float("nan")), etr.ERR_ARG), (dict(branch_scale=float("inf")), etr.ERR_ARG)])
def test_norm_configurations(change, code):
    cfg = norm_cfg(**change)
    assert etr.norm_validate(cfg) == code
    if code != etr.OK:
        n, p = C.c_size_t(0), 1 << 20
        assert etr.lib().etr_norm_workspace_bytes(C.byref(cfg), C.byref(n)) == code
        assert pointers().etr_prenorm(C.addressof(cfg), p, p, p, p, None) == code
        assert pointers().etr_join_bwd(C.addressof(cfg), *[p] * 15, None) == code


def test_norm_pointers_are_checked():
    L, cfg, ok = pointers(), norm_cfg(), 1 << 20
    a = C.addressof(cfg)
    calls = {"etr_prenorm": ("X", "w?", "N", "rstd?"),
             "etr_join": ("X", "Y", "w_post?", "gate?", "w_next?", "Xo", "N?", "rstd_y?", "rstd_o?"),
             "etr_prenorm_bwd": ("dN", "X", "w?", "rstd", "dres?", "dX", "dw?", "ws"),
             "etr_join_bwd": ("dXo?", "dN?", "Y", "Xo", "w_post?", "gate?", "w_next?", "rstd_y", "rstd_o", "dX", "dY", "dw_post?",
                              "dgate?", "dw_next?", "ws")}
    for name, args in calls.items():
        f = getattr(L, name)
        for i, arg in enumerate(args):
            assert f(a, *[ok + 4 if j == i else ok for j in range(len(args))], None) == etr.ERR_ALIGN, (name, arg)
            if not arg.endswith("?"):
                assert f(a, *[None if j == i else ok for j in range(len(args))], None) == etr.ERR_ARG, (name, arg)
    j = dict(dXo=None, dN=None, Y=ok, Xo=None, w_post=None, gate=None, w_next=None, rstd_y=ok, rstd_o=None, dX=ok, dY=ok,
             dw_post=None, dgate=None, dw_next=None, ws=None)
    assert L.etr_join_bwd(a, *j.values(), None) == etr.ERR_ARG                     # neither gradient
    assert L.etr_join_bwd(a, *dict(j, dXo=ok, dw_next=ok, ws=ok).values(), None) == etr.ERR_ARG   # dw_next without dN
    assert L.etr_join_bwd(a, *dict(j, dXo=ok, dw_post=ok).values(), None) == etr.ERR_ARG      # a gain's gradient without ws


def test_binding_refuses_what_addresses_do_not_show():
    """Tensors that are not on a GPU, or no tensors, never reach the library (types, sizes and order: the GPU tests)."""
    cfg = norm_cfg()
    x = torch.zeros(4, 16, dtype=torch.bfloat16)
    for bad in (x, None, 7):
        with pytest.raises(etr.EtrError) as e:
            etr.prenorm(cfg, bad, None, x)
        assert e.value.code == etr.ERR_ARG
    plan = etr.SortBuffers(sort_cfg(), device="cpu")
    for other in (dict(T=5), dict(k=1), dict(E=4), dict(align=2), dict(align=128, capacity=4)):
        with pytest.raises(etr.EtrError) as e:
            etr.sort_rows(sort_cfg(**other), x, plan, x)          # a plan of another configuration
        assert e.value.code in (etr.ERR_WORKSPACE, etr.ERR_ARG)
    with pytest.raises(etr.EtrError) as e:
        etr.sort(plan.cfg, torch.zeros(4, 2, dtype=torch.int32), plan)
    assert e.value.code == etr.ERR_ARG


def composed(cfg, ncfg):
    """The four composed calls with addresses that nothing is read from; a change replaces one argument by name."""
    L, ok = etr.lib(), 1 << 20
    p = C.c_void_p(ok)
    buf, n = etr.Buffers(), C.c_size_t(0)
    assert L.etr_buffers_bytes(C.byref(cfg), 0, C.byref(n)) == etr.OK
    assert L.etr_buffers_bind(C.byref(cfg), 0, p, n, C.byref(buf)) == etr.OK
    a = dict(cfg=C.byref(cfg), ncfg=C.byref(ncfg), buf=C.byref(buf), plan=C.byref(etr.SortPlan(*[ok] * 6)),
             bb=C.byref(etr.BlockBuffersC(*[ok] * 7)), stream=None)
    names = {"etr_routed_forward": "cfg X ids weights W1g W1u W2 buf plan Y stream",
             "etr_routed_backward": "cfg weights W1g W1u W2 dY buf plan dX dweights dW1g dW1u dW2 stream",
             "etr_block_forward": "cfg ncfg X w_pre? w_post? gate? R W1g W1u W2 buf bb Xo stream",
             "etr_block_backward": "cfg ncfg X w_pre? w_post? gate? R W1g W1u W2 dXo buf bb dX dw_pre? dw_post? dgate? dR dW1g dW1u dW2 stream"}

    def call(name, **change):
        return getattr(L, name)(*[change.get(x.rstrip("?"), a.get(x, p)) for x in names[name].split()])

    return names, call, buf


def test_composed_calls_check_their_arguments():
    cfg = etr.make_config(T=64, d=256, D=8, E=8, k=2, h=128, capacity=64, dtype=etr.BF16, weight_dtype=etr.F32)
    ncfg = etr.make_norm_config(T=64, d=256, dtype=etr.BF16)
    names, call, buf = composed(cfg, ncfg)
    for name, args in names.items():
        for x in args.split():
            if x in ("cfg", "ncfg", "buf", "plan", "bb", "stream"):
                if x != "stream":
                    assert call(name, **{x: None}) == etr.ERR_ARG, (name, x)
                continue
            assert call(name, **{x.rstrip("?"): C.c_void_p((1 << 20) + 4)}) == etr.ERR_ALIGN, (name, x)
            if not x.endswith("?"):
                assert call(name, **{x: None}) == etr.ERR_ARG, (name, x)
        small = etr.Buffers.from_buffer_copy(buf)
        small.ws_bytes = 16
        assert call(name, buf=C.byref(small)) == etr.ERR_WORKSPACE
        if name.startswith("etr_block"):
            for bad in (dict(T=63), dict(d=248), dict(dtype=etr.F32)):
                other = etr.make_norm_config(**dict(dict(T=64, d=256, dtype=etr.BF16), **bad))
                assert call(name, ncfg=C.byref(other)) == etr.ERR_SHAPE
    many = etr.make_config(T=64, d=512, D=8, E=64, k=33, h=128, capacity=64, dtype=etr.BF16)
    assert etr.validate(many) == etr.OK
    for name in ("etr_routed_forward", "etr_routed_backward"):
        assert composed(many, ncfg)[1](name) == etr.ERR_SHAPE


def test_block_buffers_are_carved_in_order():
    ncfg, L, n, b = etr.make_norm_config(T=65, d=264, dtype=etr.BF16), etr.lib(), C.c_size_t(0), etr.BlockBuffersC()
    assert L.etr_block_bind(C.byref(ncfg), None, 0, None, C.byref(n)) == etr.OK and n.value % 256 == 0
    assert L.etr_block_bind(C.byref(ncfg), C.c_void_p((1 << 20) + 16), n, C.byref(b), None) == etr.ERR_ALIGN
    assert L.etr_block_bind(C.byref(ncfg), C.c_void_p(1 << 20), C.c_size_t(4096), C.byref(b), None) == etr.ERR_WORKSPACE
    assert L.etr_block_bind(C.byref(ncfg), C.c_void_p(1 << 20), n, C.byref(b), None) == etr.OK
    rows = 65 * 264 * 2
    at = [getattr(b, x) for x in ("N", "Y", "dN", "dY", "rstd_x", "rstd_y", "ws")] + [(1 << 20) + n.value]
    assert all(v % 256 == 0 for v in at) and all(q - p >= s for p, q, s in zip(at, at[1:], [rows] * 4 + [260] * 2 + [etr.norm_workspace_bytes(ncfg)]))
