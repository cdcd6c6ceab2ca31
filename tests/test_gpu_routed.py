"""The layer's experts under a router's own choice: what the capacity does to choices that name an expert twice."""
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
