"""The row operators as they are used: the layer's experts under a router of the caller's own, and the norm, layer and join of a
block, forward and backward, against torch autograd in 64 bits and against the layer's own path."""
import numpy as np
import pytest
import torch

from gen import workloads as gw
from paper_2406_00023_b200 import etr
from tests import harness as hz
from tests import rows_reference as rr

pytestmark = pytest.mark.gpu
EPS = 1e-6


def ffn64(x, W1g, W1u, W2):
    g, u = x @ W1g.T, x @ W1u.T
    return (torch.nn.functional.silu(g) * u) @ W2.T


def routed64(X, ids, w, W1g, W1u, W2, capacity):
    """Sum over a token's choices of weight * expert, pairs behind an expert's first `capacity` left out."""
    Y = torch.zeros_like(X)
    for e in range(W1g.shape[0]):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        t, j = t[:capacity], j[:capacity]
        if t.numel():
            Y = Y.index_add(0, t, w[t, j][:, None] * ffn64(X[t], W1g[e], W1u[e], W2[e]))
    return Y


def inputs(T, d, h, E, k, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device="cuda") * scale).to(dtype)       # noqa: E731
    x = dict(X=rand(T, d), dY=rand(T, d), W1g=rand(E, h, d, scale=d ** -0.5), W1u=rand(E, h, d, scale=d ** -0.5),
             W2=rand(E, d, h, scale=d ** -0.5))
    score = torch.randn(T, E, generator=g, device="cuda") + torch.randn(E, generator=g, device="cuda")
    top = torch.topk(score, k)
    ids = top.indices.to(torch.int32)
    ids[torch.rand(T, generator=g, device="cuda") < 0.1] = -1
    if k > 1:
        ids[0, 1] = ids[0, 0]                              # one token names an expert twice
    return x, ids.contiguous(), torch.softmax(top.values, 1).contiguous()


def close(got, ref, dtype, what, chain):
    """fp32: |err| <= 1e-4 rms(ref) element by element.  bf16: rms(err) <= 2e-3 sqrt(chain) rms(ref).  A value rounded to bf16 is
    off by an error uniform within half a step, 2^-8 of a value at the low end of its binade and 2^-9 at the high end: an RMS
    of 2^-8 sqrt(avg of m^-2 over a mantissa m spread evenly in [1, 2)) / sqrt(3) = 2^-8 sqrt(1/2) / sqrt(3) = 1.6e-3 of the
    value; `chain` such errors add up incoherently.  (The harness's element-wise statements for bf16 count outliers of sums over
    hundreds of rows an expert, more than there are here; that bf16 values are right one by one follows from the stage
    tests and from test_composed_calls_are_their_stages.)"""
    got, ref = hz.to_np(got), ref.float().cpu().numpy()
    if dtype == torch.float32:
        hz.assert_close_rms(got, ref, 1e-4, what, chain=chain)
    else:
        assert hz.error_stats(got, ref)[1] <= 2e-3 * np.sqrt(chain), (what, hz.error_stats(got, ref))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T, d, h, E, k, cap", [(300, 256, 192, 8, 2, "all"), (700, 512, 256, 12, 3, "cut"), (1, 256, 64, 4, 1, "all"),
                                                (129, 320, 128, 16, 8, "all")])
def test_experts_under_a_given_choice(T, d, h, E, k, cap, dtype):
    x, ids, w = inputs(T, d, h, E, k, dtype, T)
    capacity = 2 * T if cap == "all" else max(1, T * k // E // 2)
    cfg = etr.make_config(T=T, d=d, D=8, E=E, k=k, h=h, capacity=capacity, dtype=etr.F32 if dtype == torch.float32 else etr.BF16)
    buf, plan = etr.LayerBuffers(cfg), etr.SortBuffers(etr.routed_sort_config(cfg))
    W = (x["W1g"], x["W1u"], x["W2"])
    Y, dX, dw = torch.empty_like(x["X"]), torch.empty_like(x["X"]), torch.empty_like(w)
    dW = [torch.empty_like(t) for t in W]
    for _ in range(2):                                     # the second pass finds the first one's buffers
        etr.routed_forward(cfg, x["X"], ids, w, *W, buf, plan, Y)
        etr.routed_backward(cfg, w, *W, x["dY"], buf, plan, dX, dw, *dW)
    assert buf.read_stats().error_word == 0
    leaves = [t.double().requires_grad_() for t in (x["X"], w, *W)]
    ref = routed64(leaves[0], ids, leaves[1], *leaves[2:], capacity)
    grads = torch.autograd.grad(ref, leaves, x["dY"].double())
    close(Y, ref.detach(), dtype, "Y", 4)
    for name, got, want, chain in (("dX", dX, grads[0], 6), ("dweights", dw, grads[1], 4), ("dW1g", dW[0], grads[2], 6),
                                   ("dW1u", dW[1], grads[3], 6), ("dW2", dW[2], grads[4], 4)):
        close(got, want, dtype, name, chain)


@pytest.mark.parametrize("k", [1, 2])
def test_given_choice_repeats_the_layers_own(k):
    """Token choice without a drop, its experts and affinities given back: the experts see the same rows and give the same
    bits; the sums over a token's two experts differ in their order alone."""
    w = gw.scaled(gw.WORKLOADS["small"], T=1000, k=k, cf=8.0)
    x = gw.make_inputs(w)
    dev = hz.upload(w, x)
    cfg = hz.make_cfg(w, mode=None, fuse_combine=etr.FUSE_OFF)
    buf = etr.LayerBuffers(cfg)
    W = (dev.W1g, dev.W1u, dev.W2)
    Y, dX, dR = torch.empty_like(dev.X), torch.empty_like(dev.X), torch.empty_like(dev.R)
    dW = [torch.empty_like(t) for t in W]
    etr.layer_forward(cfg, dev.X, dev.R, *W, buf, Y)
    etr.layer_backward(cfg, dev.X, dev.R, *W, dev.dY, buf, dX, dR, *dW)
    assert buf.read_stats().dropped == 0
    ids = buf.topk_idx.clone()
    weights = torch.gather(buf.delta, 1, ids.long()).contiguous()
    buf2, plan = etr.LayerBuffers(cfg), etr.SortBuffers(etr.routed_sort_config(cfg))
    Y2, dX2, dw = torch.empty_like(Y), torch.empty_like(dX), torch.empty_like(weights)
    dW2 = [torch.empty_like(t) for t in W]
    etr.routed_forward(cfg, dev.X, ids, weights, *W, buf2, plan, Y2)
    etr.routed_backward(cfg, weights, *W, dev.dY, buf2, plan, dX2, dw, *dW2)
    torch.cuda.synchronize()
    assert torch.equal(plan.counts, buf.counts) and torch.equal(plan.row_token, buf.slot_token)
    live = buf.slot_token >= 0
    for n in ("Xp", "G", "U", "H", "O", "dO", "dG", "dU", "dXp"):
        assert torch.equal(getattr(buf, n)[live], getattr(buf2, n)[live]), n
    for a, b in zip(dW, dW2):
        assert torch.equal(a, b)
    assert torch.equal(Y, Y2) if k == 1 else True
    rr.assert_within(Y2, *rr.unsort(buf.O, weights, plan.pos, torch.bfloat16), "Y")
    rr.assert_within(dX2, *rr.unsort(buf.dXp, None, plan.pos, torch.bfloat16), "dX")
    rows = plan.pos.long()
    got = dw.double()
    rr.assert_within(got, buf.dgate.double()[rows], (2 * w.d + 2) * rr.U * (dev.dY.double()[:, None] * buf.O.double()[rows]).abs().sum(2), "dweights")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T, d, h, E, k, cap", [(129, 320, 128, 16, 8, "all"), (700, 512, 256, 12, 3, "cut")])
def test_composed_calls_are_their_stages(T, d, h, E, k, cap, dtype):
    """etr_routed_forward and _backward, bit for bit the stage calls in a row."""
    x, ids, w = inputs(T, d, h, E, k, dtype, T + 1)
    cfg = etr.make_config(T=T, d=d, D=8, E=E, k=k, h=h, capacity=2 * T if cap == "all" else max(1, T * k // E // 2),
                          dtype=etr.F32 if dtype == torch.float32 else etr.BF16)
    W = (x["W1g"], x["W1u"], x["W2"])
    res = []
    for composed in (True, False):
        sc = etr.routed_sort_config(cfg)
        b, plan = etr.LayerBuffers(cfg), etr.SortBuffers(sc)
        Y, dX, dw, dW = torch.empty_like(x["X"]), torch.empty_like(x["X"]), torch.empty_like(w), [torch.empty_like(t) for t in W]
        if composed:
            etr.routed_forward(cfg, x["X"], ids, w, *W, b, plan, Y)
            etr.routed_backward(cfg, w, *W, x["dY"], b, plan, dX, dw, *dW)
        else:
            b.stats.zero_()
            ws = torch.empty(etr.workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
            etr.sort(sc, ids, plan)
            etr.sort_rows(sc, x["X"], plan, b.Xp)
            b.counts.copy_(plan.counts)
            b.slot_token.copy_(plan.row_token)
            etr.expert_ffn(cfg, b.route, b.Xp, *W, b.G, b.U, b.H, b.O, b.c.stats, ws)
            etr.unsort_rows(sc, b.O, w, plan, Y)
            etr.unsort_rows_bwd(sc, x["dY"], b.O, w, plan, b.dO, dw)
            etr.expert_ffn_bwd(cfg, b.route, b.dO, b.Xp, b.G, b.U, b.H, *W, b.dG, b.dU, b.dXp, *dW, b.c.stats, ws)
            etr.sort_rows_bwd(sc, b.dXp, plan, dX)
        torch.cuda.synchronize()
        res.append([Y, dX, dw, *dW])
    assert all(torch.equal(p, q) for p, q in zip(*res))


@pytest.mark.parametrize("gemm", [etr.GEMM_TCGEN05, etr.GEMM_TCGEN05_2CTA, etr.GEMM_TCGEN05_2CTA_WIDE, etr.GEMM_SIMT])
def test_given_choice_in_every_gemm_form(gemm):
    T, d, h, E, k = 400, 512, 256, 8, 2
    x, ids, w = inputs(T, d, h, E, k, torch.bfloat16, 3)
    outs = []
    for impl in (etr.GEMM_AUTO, gemm):
        cfg = etr.make_config(T=T, d=d, D=8, E=E, k=k, h=h, capacity=T, dtype=etr.BF16, gemm_impl=impl)
        buf, plan = etr.LayerBuffers(cfg), etr.SortBuffers(etr.routed_sort_config(cfg))
        Y = torch.empty_like(x["X"])
        etr.routed_forward(cfg, x["X"], ids, w, x["W1g"], x["W1u"], x["W2"], buf, plan, Y)
        assert buf.read_stats().error_word == 0
        outs.append(Y)
    close(outs[1], outs[0], torch.bfloat16, "Y", 4)


def test_given_choice_with_fp32_master_weights():
    T, d, h, E, k = 400, 512, 256, 8, 2
    x, ids, w = inputs(T, d, h, E, k, torch.bfloat16, 4)
    kw = dict(T=T, d=d, D=8, E=E, k=k, h=h, capacity=T, dtype=etr.BF16)
    res = []
    for cfg, up in ((etr.make_config(**kw, grad_fp32=True), False), (etr.make_config(**kw, weight_dtype=etr.F32), True)):
        W = [x[n].float() if up else x[n] for n in ("W1g", "W1u", "W2")]
        buf, plan = etr.LayerBuffers(cfg), etr.SortBuffers(etr.routed_sort_config(cfg))
        Y, dX, dw, dW = torch.empty_like(x["X"]), torch.empty_like(x["X"]), torch.empty_like(w), [torch.empty_like(t, dtype=torch.float32) for t in W]
        etr.routed_forward(cfg, x["X"], ids, w, *W, buf, plan, Y)
        etr.routed_backward(cfg, w, *W, x["dY"], buf, plan, dX, dw, *dW)
        torch.cuda.synchronize()
        res.append([Y, dX, dw, *dW])
    assert all(torch.equal(a, b) for a, b in zip(*res))


@pytest.mark.parametrize("name, post, gated", [("tiny", True, True), ("tiny", False, False), ("small", True, True), ("small", True, False)])
def test_block_is_norm_layer_join(name, post, gated):
    """Bit for bit the three calls by themselves, each way."""
    w = gw.scaled(gw.WORKLOADS[name], T=512)
    x = gw.make_inputs(w)
    dev = hz.upload(w, x)
    cfg = hz.make_cfg(w)
    n = etr.make_norm_config(T=w.T, d=w.d, dtype=cfg.dtype, eps=EPS, res_scale=0.875, branch_scale=0.5, post_norm=post)
    g = torch.Generator(device="cuda").manual_seed(5)
    w_pre, w_post = (1 + 0.2 * torch.randn(w.d, generator=g, device="cuda") for _ in range(2))
    gate = torch.rand(w.T, generator=g, device="cuda") if gated else None
    W, f32 = (dev.W1g, dev.W1u, dev.W2), dict(dtype=torch.float32, device="cuda")

    def grads():
        return dict(dX=torch.empty_like(dev.X), dw_pre=torch.empty(w.d, **f32), dw_post=torch.empty(w.d, **f32),
                    dgate=torch.empty(w.T, **f32) if gated else None, dR=torch.empty_like(dev.R), dW1g=torch.empty_like(dev.W1g),
                    dW1u=torch.empty_like(dev.W1u), dW2=torch.empty_like(dev.W2))

    buf, bb, Xo, a = etr.LayerBuffers(cfg), etr.BlockBuffers(n), torch.empty_like(dev.X), grads()
    etr.block_forward(cfg, n, dev.X, w_pre, w_post, gate, dev.R, *W, buf, bb, Xo)
    etr.block_backward(cfg, n, dev.X, w_pre, w_post, gate, dev.R, *W, dev.dY, buf, bb, *a.values())
    assert buf.read_stats().error_word == 0
    buf, b = etr.LayerBuffers(cfg), grads()
    N, Y, Xo2, dY, dN, dXa = (torch.empty_like(dev.X) for _ in range(6))
    rx, ry = torch.empty(w.T, **f32), torch.empty(w.T, **f32)
    ws = torch.empty(etr.norm_workspace_bytes(n), dtype=torch.uint8, device="cuda")
    etr.prenorm(n, dev.X, w_pre, N, rx)
    etr.layer_forward(cfg, N, dev.R, *W, buf, Y)
    etr.join(n, dev.X, Y, w_post, gate, None, Xo2, None, ry)
    etr.join_bwd(n, dev.dY, None, Y, None, w_post, gate, None, ry, None, dXa, dY, b["dw_post"], b["dgate"], None, ws)
    etr.layer_backward(cfg, N, dev.R, *W, dY, buf, dN, b["dR"], b["dW1g"], b["dW1u"], b["dW2"])
    etr.prenorm_bwd(n, dN, dev.X, w_pre, rx, dXa, b["dX"], b["dw_pre"], ws)
    torch.cuda.synchronize()
    assert torch.equal(Xo, Xo2)
    for key in a:
        assert a[key] is None or torch.equal(a[key], b[key]), key
    # and the sum is what the definition says of the layer's own output
    rr.assert_within(Xo, *rr.join(dev.X, Y, w_post, gate, None, EPS, 0.875, 0.5, post, dev.X.dtype)["Xo"], "Xo")


def test_two_blocks_with_a_router_of_their_own():
    """A residual stream through two blocks of experts under a router's choice, the second block's norm joined to the first one's
    end; all gradients against autograd in 64 bits with the choice held constant.  fp32: its errors stay far below 1e-4 however
    they pass through the SwiGLUs."""
    dtype = torch.float32
    T, d, h, E, k, a, b = 257, 256, 128, 8, 2, 0.875, 0.5
    code = etr.F32
    g = torch.Generator(device="cuda").manual_seed(11)
    rand = lambda *s, scale=1.0, t=dtype: (torch.randn(*s, generator=g, device="cuda") * scale).to(t)     # noqa: E731
    f32 = torch.float32
    X0, dXo = rand(T, d), rand(T, d)
    ids = [torch.topk(torch.randn(T, E, generator=g, device="cuda"), k).indices.to(torch.int32).contiguous() for _ in range(2)]
    wts = [torch.softmax(torch.randn(T, k, generator=g, device="cuda"), 1).contiguous() for _ in range(2)]
    W = [[rand(E, h, d, scale=d ** -0.5), rand(E, h, d, scale=d ** -0.5), rand(E, d, h, scale=d ** -0.5)] for _ in range(2)]
    pre, post = ([1 + rand(d, scale=0.2, t=f32) for _ in range(2)] for _ in range(2))
    gate = [torch.rand(T, generator=g, device="cuda") for _ in range(2)]
    cfg = etr.make_config(T=T, d=d, D=8, E=E, k=k, h=h, capacity=T, dtype=code)
    n = etr.make_norm_config(T=T, d=d, dtype=code, eps=EPS, res_scale=a, branch_scale=b, post_norm=True)
    bufs, plans = [etr.LayerBuffers(cfg) for _ in range(2)], [etr.SortBuffers(etr.routed_sort_config(cfg)) for _ in range(2)]
    act, row = (lambda: torch.empty(T, d, dtype=dtype, device="cuda")), (lambda: torch.empty(T, device="cuda"))
    N, Y, X, ry, ro = [act(), act()], [act(), act()], [X0, act(), act()], [row(), row()], [row(), row()]
    etr.prenorm(n, X0, pre[0], N[0], ro[0])
    for i in range(2):
        etr.routed_forward(cfg, N[i], ids[i], wts[i], *W[i], bufs[i], plans[i], Y[i])
        last = i == 1
        etr.join(n, X[i], Y[i], post[i], gate[i], None if last else pre[1], X[i + 1], None if last else N[1], ry[i], None if last else ro[1])
    ws = torch.empty(etr.norm_workspace_bytes(n), dtype=torch.uint8, device="cuda")
    out, stream, dN, dY = {}, dXo.clone(), act(), act()
    for i in (1, 0):
        last = i == 1
        out["post", i], out["gate", i], dwn = torch.empty(d, device="cuda"), row(), None if last else torch.empty(d, device="cuda")
        etr.join_bwd(n, stream, None if last else dN, Y[i], None if last else X[1], post[i], gate[i], None if last else pre[1], ry[i],
                     None if last else ro[1], stream, dY, out["post", i], out["gate", i], dwn, ws)
        if not last:
            out["pre", 1] = dwn
        out["wts", i], dW = torch.empty_like(wts[i]), [torch.empty_like(t) for t in W[i]]
        etr.routed_backward(cfg, wts[i], *W[i], dY, bufs[i], plans[i], dN, out["wts", i], *dW)
        for j in range(3):
            out["W", i, j] = dW[j]
    out["pre", 0] = torch.empty(d, device="cuda")
    etr.prenorm_bwd(n, dN, X0, pre[0], ro[0], stream, stream, out["pre", 0], ws)
    torch.cuda.synchronize()
    out["X"] = stream
    leaf = {"X": X0}
    for i in range(2):
        leaf.update({("pre", i): pre[i], ("post", i): post[i], ("gate", i): gate[i], ("wts", i): wts[i]})
        leaf.update({("W", i, j): W[i][j] for j in range(3)})
    leaf = {key: t.double().requires_grad_() for key, t in leaf.items()}
    norm = lambda x, w: x * (x.square().mean(1, keepdim=True) + EPS).rsqrt() * w                          # noqa: E731
    x = leaf["X"]
    for i in range(2):
        y = routed64(norm(x, leaf["pre", i]), ids[i], leaf["wts", i], *[leaf["W", i, j] for j in range(3)], T)
        x = a * x + b * leaf["gate", i][:, None] * norm(y, leaf["post", i])
    grads = dict(zip(leaf, torch.autograd.grad(x, list(leaf.values()), dXo.double())))
    close(X[2], x.detach(), dtype, "Xo", 12)                # N, H, O, Y, Xo of each block and what they are made of
    for key in out:
        close(out[key], grads[key], dtype, str(key), 20)    # both passes' stores of both blocks


def test_captured_block_follows_its_inputs():
    w = gw.scaled(gw.WORKLOADS["small"], T=512)
    dev = hz.upload(w, gw.make_inputs(w))
    cfg = hz.make_cfg(w)
    n = etr.make_norm_config(T=w.T, d=w.d, dtype=cfg.dtype, post_norm=True)
    buf, bb, Xo = etr.LayerBuffers(cfg), etr.BlockBuffers(n), torch.empty_like(dev.X)
    ids, wt, plan, Y = torch.zeros(w.T, w.k, dtype=torch.int32, device="cuda"), torch.rand(w.T, w.k, device="cuda"), etr.SortBuffers(etr.routed_sort_config(cfg)), torch.empty_like(dev.X)

    def calls():
        etr.block_forward(cfg, n, dev.X, None, None, None, dev.R, dev.W1g, dev.W1u, dev.W2, buf, bb, Xo)
        etr.routed_forward(cfg, Xo, ids, wt, dev.W1g, dev.W1u, dev.W2, buf, plan, Y)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    dev.X.copy_(torch.randn_like(dev.X))
    ids.copy_(torch.randint(0, w.E, ids.shape))
    graph.replay()
    torch.cuda.synchronize()
    replayed = Xo.clone(), Y.clone()
    calls()
    torch.cuda.synchronize()
    assert torch.equal(Xo, replayed[0]) and torch.equal(Y, replayed[1])


def test_two_streams_at_once():
    """Calls on two streams with buffers of their own, interleaved without a wait between them: the bits of either alone."""
    T, d, E, k = 5000, 1024, 48, 3
    g = torch.Generator(device="cuda").manual_seed(6)
    sc = etr.make_sort_config(T=T, k=k, E=E, d=d, dtype=etr.BF16, align=8)
    nc = etr.make_norm_config(T=T, d=d, dtype=etr.BF16, eps=EPS, post_norm=True)
    sets = []
    for _ in range(2):
        x = dict(ids=torch.randint(0, E, (T, k), generator=g, device="cuda", dtype=torch.int32), w=torch.rand(T, k, generator=g, device="cuda"),
                 gain=torch.rand(d, generator=g, device="cuda"), gate=torch.rand(T, generator=g, device="cuda"))
        for n in ("X", "dY", "dX"):
            x[n] = torch.randn(T, d, generator=g, device="cuda").bfloat16()
        sets.append(x)

    def state():
        plan = etr.SortBuffers(sc)
        rows = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")                            # noqa: E731
        return dict(plan=plan, N=rows(T, d), Xs=rows(plan.n_rows, d), Y=rows(T, d), Xo=rows(T, d), dYo=rows(T, d), dXo=rows(T, d),
                    dO=rows(plan.n_rows, d), dw=torch.zeros(T, k, device="cuda"), r=torch.zeros(T, device="cuda"), ry=torch.zeros(T, device="cuda"),
                    dgain=torch.zeros(d, device="cuda"), ws=torch.empty(etr.norm_workspace_bytes(nc), dtype=torch.uint8, device="cuda"))

    def step(x, s):
        etr.prenorm(nc, x["X"], x["gain"], s["N"], s["r"])
        etr.sort(sc, x["ids"], s["plan"])
        etr.sort_rows(sc, s["N"], s["plan"], s["Xs"])
        etr.unsort_rows(sc, s["Xs"], x["w"], s["plan"], s["Y"])
        etr.join(nc, x["X"], s["Y"], x["gain"], x["gate"], None, s["Xo"], None, s["ry"])
        etr.join_bwd(nc, x["dX"], None, s["Y"], None, x["gain"], x["gate"], None, s["ry"], None, s["dXo"], s["dYo"], s["dgain"], None, None, s["ws"])
        etr.unsort_rows_bwd(sc, s["dYo"], s["Xs"], x["w"], s["plan"], s["dO"], s["dw"])

    names = ("N", "Xs", "Y", "Xo", "dYo", "dXo", "dO", "dw", "dgain")
    alone = []
    for x in sets:
        s = state()
        step(x, s)
        torch.cuda.synchronize()
        alone.append({n: s[n].clone() for n in names})
    both, streams = [state(), state()], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for x, s, stream in zip(sets, both, streams):
            with torch.cuda.stream(stream):
                step(x, s)
    torch.cuda.synchronize()
    for s, ref in zip(both, alone):
        for n in names:
            assert torch.equal(s[n], ref[n]), n
