"""The largest values that the norm and the join take, in the widest rows: 16384 squares of 1e17 come to half of what fp32 holds."""
import pytest
import torch

from paper_2406_00023_b200 import etr
from tests import rows_reference as rr

pytestmark = pytest.mark.gpu
T, D, EPS, TOP = 6, 16384, 1e-6, 9.9e16
TYPES = pytest.mark.parametrize("dtype, code", [(torch.bfloat16, etr.BF16), (torch.float32, etr.F32)], ids=["bf16", "f32"])


def spread(dtype, g, size=TOP):
    """Rows up to `size`, the first one of nothing else."""
    x = (torch.rand(T, D, generator=g, device="cuda") * 2 - 1) * size
    x[0] = size
    return x.to(dtype)


def nans(*shape, dtype=torch.float32):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


@TYPES
@pytest.mark.parametrize("post", [True, False])
def test_join_at_the_documented_size(dtype, code, post):
    """Half of X and half of Y come to a sum of the documented size without the post norm; with it the branch is of the gains' size,
    so X alone makes the sum (a = 1)."""
    g = torch.Generator(device="cuda").manual_seed(7)
    a, b = (1.0, 0.5) if post else (0.5, 0.5)
    cfg = etr.make_norm_config(T=T, d=D, dtype=code, eps=EPS, res_scale=a, branch_scale=b, post_norm=post)
    X, Y = spread(dtype, g), spread(dtype, g)
    w_post = 1 - 0.3 * torch.rand(D, generator=g, device="cuda")
    w_next = 1 + 0.3 * torch.randn(D, generator=g, device="cuda")
    gate = torch.rand(T, generator=g, device="cuda")
    w_post[:100], gate[0] = 1.0, 1.0
    Xo, N, ry, ro = nans(T, D, dtype=dtype), nans(T, D, dtype=dtype), nans(T), nans(T)
    etr.join(cfg, X, Y, w_post, gate, w_next, Xo, N, ry, ro)
    ref = rr.join(X, Y, w_post, gate, w_next, EPS, a, b, post, dtype)
    for name, got in (("Xo", Xo), ("N", N), ("rstd_o", ro)) + ((("rstd_y", ry),) if post else ()):
        rr.assert_within(got, *ref[name], name)


@TYPES
@pytest.mark.parametrize("post", [True, False])
def test_join_gradients_at_the_documented_size(dtype, code, post):
    g = torch.Generator(device="cuda").manual_seed(8)
    a, b = 0.875, 0.5
    cfg = etr.make_norm_config(T=T, d=D, dtype=code, eps=EPS, res_scale=a, branch_scale=b, post_norm=post)
    Y, Xo, dXo = spread(dtype, g), spread(dtype, g), spread(dtype, g, TOP / 2)
    w_post, w_next = (1 + 0.5 * torch.rand(D, generator=g, device="cuda") for _ in range(2))
    dN = spread(dtype, g, TOP / 1.5)                       # times w_next: up to TOP
    # rows near zero, whose 1/rms is 1000: the gradients times that stay at the documented size
    Y[2], dXo[2], dN[2] = Y[2].float() * 1e-30, dXo[2].float() * 1e-3, dN[2].float() * 1e-3
    Xo[3], dXo[3], dN[3] = Xo[3].float() * 1e-30, dXo[3].float() * 1e-3, dN[3].float() * 1e-4
    gate = torch.rand(T, generator=g, device="cuda")
    ry, ro = (rr.prenorm(x, None, EPS, dtype)[1][0].float() for x in (Y, Xo))
    out = dict(dX=nans(T, D, dtype=dtype), dY=nans(T, D, dtype=dtype), dw_post=nans(D), dgate=nans(T), dw_next=nans(D))
    ws = torch.empty(etr.norm_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    etr.join_bwd(cfg, dXo, dN, Y, Xo, w_post, gate, w_next, ry if post else None, ro, *out.values(), ws)
    ref = rr.join_bwd(dXo, dN, Y, Xo, w_post, gate, w_next, ry, ro, a, b, post, dtype)
    for name in out:
        assert bool(ref[name][0].isfinite().all())
        rr.assert_within(out[name], *ref[name], name)
