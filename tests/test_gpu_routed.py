"""The layer's experts under a router's own choice: what the capacity does to choices that name an expert twice, and what the composed
calls refuse before a launch."""
import pytest
import torch

from paper_2406_00023_b200 import etr
from tests import rows_reference as rr

pytestmark = pytest.mark.gpu


def layer(T, d, h, E, k, capacity, dtype=etr.F32, seed=1, **kw):
    """A configuration, its buffers, a plan and random tensors of every argument."""
    cfg = etr.make_config(T=T, d=d, D=8, E=E, k=k, h=h, capacity=capacity, dtype=dtype, **kw)
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s, scale=1.0: (torch.randn(*s, generator=g, device="cuda") * scale).to(etr.torch_dtype(cfg))       # noqa: E731
    W = [rand(E, h, d, scale=d ** -0.5), rand(E, h, d, scale=d ** -0.5), rand(E, d, h, scale=h ** -0.5)]
    return cfg, etr.LayerBuffers(cfg), etr.SortBuffers(etr.routed_sort_config(cfg)), rand(T, d), torch.rand(T, k, generator=g, device="cuda"), W


@pytest.mark.parametrize("k", [2, 3])
def test_capacity_for_choices_that_repeat_an_expert(k):
    """Every token names expert 1 k times: T rows hold every pair only where no token names an expert twice, k T rows always do."""
    T, d, h, E = 200, 128, 64, 4
    same = torch.ones(T, k, dtype=torch.int32, device="cuda")
    other = torch.arange(k, dtype=torch.int32, device="cuda").repeat(T, 1).contiguous()
    for ids, capacity, dropped in ((same, T, (k - 1) * T), (same, k * T, 0), (other, T, 0)):
        cfg, buf, plan, X, w, W = layer(T, d, h, E, k, capacity)
        Y = torch.empty_like(X)
        etr.routed_forward(cfg, X, ids, w, *W, buf, plan, Y)
        assert plan.totals.tolist() == [k * T - dropped, dropped, 0, 0]
        want = rr.plan(ids, E, 128, capacity, plan.n_rows)
        assert plan.counts.tolist() == want[0] and plan.pos.tolist() == want[4]
        rr.assert_within(Y, *rr.unsort(buf.O, w, plan.pos, X.dtype), "Y")
        x64, kept = X.double(), (plan.pos >= 0).double() * w.double()
        ref = torch.zeros_like(x64)
        for e in range(E):
            g, u, o = (t[e].double() for t in W)
            ref += (kept * (ids == e)).sum(1, keepdim=True) * ((torch.nn.functional.silu(x64 @ g.T) * (x64 @ u.T)) @ o.T)
        # fp32 contractions of 128 and 64 terms and a SwiGLU between them, each off by less than 1e-5 of its own RMS
        assert float((Y.double() - ref).abs().max()) <= 1e-4 * float(ref.square().mean().sqrt())


def everything(dtype=etr.BF16, **kw):
    """Arguments of the four composed calls by name, all of them right."""
    T, d, h, E, k = 48, 256, 64, 8, 2
    cfg, buf, plan, X, w, W = layer(T, d, h, E, k, T, dtype, **kw)
    n = etr.make_norm_config(T=T, d=d, dtype=dtype, post_norm=True)
    act, f32 = (lambda: torch.zeros_like(X)), (lambda *s: torch.ones(*s, device="cuda"))
    W = [t.to(torch.float32 if cfg.weight_dtype == etr.F32 else torch.bfloat16) for t in W]
    grad = torch.float32 if cfg.grad_fp32 or cfg.weight_dtype == etr.F32 else torch.bfloat16
    a = dict(cfg=cfg, ncfg=n, buf=buf, plan=plan, bb=etr.BlockBuffers(n), X=X, topk_idx=torch.zeros(T, k, dtype=torch.int32, device="cuda"),
             weights=w, W1g=W[0], W1u=W[1], W2=W[2], Y=act(), dY=act(), dX=act(), dweights=f32(T, k), Xo=act(), dXo=act(), w_pre=f32(d),
             w_post=f32(d), gate=f32(T), R=torch.randn(E, d // 8, device="cuda"), dw_pre=f32(d), dw_post=f32(d), dgate=f32(T), dR=f32(E, d // 8))
    a.update({"d" + name: torch.zeros_like(a[name], dtype=grad) for name in ("W1g", "W1u", "W2")})
    names = {"routed_forward": "cfg X topk_idx weights W1g W1u W2 buf plan Y",
             "routed_backward": "cfg weights W1g W1u W2 dY buf plan dX dweights dW1g dW1u dW2",
             "block_forward": "cfg ncfg X w_pre w_post gate R W1g W1u W2 buf bb Xo",
             "block_backward": "cfg ncfg X w_pre w_post gate R W1g W1u W2 dXo buf bb dX dw_pre dw_post dgate dR dW1g dW1u dW2"}
    return a, {name: args.split() for name, args in names.items()}


MAY_BE_LEFT_OUT = {"w_pre", "w_post", "gate", "dw_pre", "dw_post", "dgate"}


@pytest.mark.parametrize("kw", [dict(), dict(dtype=etr.F32), dict(grad_fp32=True), dict(weight_dtype=etr.F32)], ids=str)
def test_composed_calls_look_every_tensor_over(kw):
    """One argument at a time: of another type (ids as torch.topk gives them among them), too short, too long, transposed, on the
    host, or left out."""
    a, names = everything(**kw)
    for name, args in names.items():
        getattr(etr, name)(*[a[x] for x in args])
    torch.cuda.synchronize()
    n0 = etr.launch_count()
    for name, args in names.items():
        for x in args:
            t = a[x]
            if not isinstance(t, torch.Tensor):
                continue
            wrong = {torch.int32: torch.int64, torch.float32: torch.bfloat16, torch.bfloat16: torch.float32}[t.dtype]
            longer = torch.zeros(t.numel() + 8, dtype=t.dtype, device="cuda")
            bad = [(t.to(wrong), etr.ERR_ARG, "of another type"), (longer, etr.ERR_SHAPE, "of another size"),
                   (longer[:t.numel() - 8], etr.ERR_SHAPE, "of another size"), (t.cpu(), etr.ERR_ARG, "not on a CUDA device")]
            if t.dim() > 1:
                bad.append((t.transpose(-1, -2), etr.ERR_SHAPE, "not contiguous"))
            if x not in MAY_BE_LEFT_OUT:
                bad.append((None, etr.ERR_ARG, "a tensor is wanted"))
            for b, code, said in bad:
                with pytest.raises(etr.EtrError) as e:
                    getattr(etr, name)(*[b if y == x else a[y] for y in args])
                assert e.value.code == code and f"etr_{name}: {x}: {said}" in str(e.value), (x, said, str(e.value))
    assert etr.launch_count() == n0
    for name, args in names.items():
        getattr(etr, name)(*[None if x in MAY_BE_LEFT_OUT else a[x] for x in args])
    torch.cuda.synchronize()


def test_buffers_of_a_larger_layer_serve_a_smaller_one():
    a, names = everything()
    big = etr.LayerBuffers(etr.make_config(T=100, d=512, D=8, E=16, k=4, h=128, capacity=300, dtype=etr.BF16))
    big.block.fill_(0x5a)
    out = []
    for buf in (a["buf"], big):
        for name, args in names.items():
            getattr(etr, name)(*[buf if x == "buf" else a[x] for x in args])
        torch.cuda.synchronize()
        out.append([a[x].clone() for x in ("Y", "Xo", "dX", "dweights", "dW1g", "dW2", "dR", "dw_pre")])
    assert all(torch.equal(p, q) for p, q in zip(*out))


def test_routed_calls_use_nothing_of_the_layers_own_router():
    """Buffers whose members of the batch's length are too short for the layer's own call, but whose rows suffice."""
    a, names = everything()
    short = etr.LayerBuffers(etr.make_config(T=8, d=256, D=32, E=8, k=1, h=64, capacity=48, dtype=etr.BF16))
    short.block.fill_(0x5a)
    out = []
    for buf in (a["buf"], short):
        for name in ("routed_forward", "routed_backward"):
            getattr(etr, name)(*[buf if x == "buf" else a[x] for x in names[name]])
        torch.cuda.synchronize()
        out.append([a[x].clone() for x in ("Y", "dX", "dweights", "dW1g", "dW1u", "dW2")])
    assert all(torch.equal(p, q) for p, q in zip(*out))
    for name in ("block_forward", "block_backward"):
        with pytest.raises(etr.EtrError) as e:
            getattr(etr, name)(*[short if x == "buf" else a[x] for x in names[name]])
        assert e.value.code == etr.ERR_WORKSPACE
