"""Calls of the row operators that are refused before a launch: by the Python binding, and by the library for members of its structs.
There is no GPU here: a launch, or a copy, would fail with another status."""
import ctypes as C

import pytest
import torch

from paper_2406_00023_b200 import etr
from tests.test_rows_reference import composed


def sort_calls(cfg, plan):
    """Every operator that takes a plan, on tensors of the right types and sizes."""
    R, bf = plan.n_rows, torch.bfloat16
    x, rows, w = torch.zeros(cfg.T, cfg.d, dtype=bf), torch.zeros(R, cfg.d, dtype=bf), torch.zeros(cfg.T, cfg.k)
    ids = torch.zeros(cfg.T, cfg.k, dtype=torch.int32)
    return {"etr_sort": lambda c: etr.sort(c, ids, plan), "etr_sort_rows": lambda c: etr.sort_rows(c, x, plan, rows),
            "etr_sort_rows_bwd": lambda c: etr.sort_rows_bwd(c, rows, plan, x), "etr_unsort_rows": lambda c: etr.unsort_rows(c, rows, w, plan, x),
            "etr_unsort_rows_bwd": lambda c: etr.unsort_rows_bwd(c, x, rows, w, plan, rows, w)}


def refused(call, code, *said):
    with pytest.raises(etr.EtrError) as e:
        call()
    assert e.value.code == code and all(s in str(e.value) for s in said), str(e.value)


def test_a_plan_that_is_not_on_a_gpu_is_refused_for_itself():
    """Whatever the tensors: the kernels would write through its addresses."""
    cfg = etr.make_sort_config(T=4, k=2, E=3, d=16, dtype=etr.BF16)
    plan = etr.SortBuffers(cfg, device="cpu")
    assert plan.device == -1
    for name, call in sort_calls(cfg, plan).items():
        refused(lambda: call(cfg), etr.ERR_ARG, name, "plan: not on a CUDA device")


@pytest.mark.parametrize("other", [dict(T=5), dict(k=1), dict(E=4), dict(align=2), dict(align=128, capacity=4)], ids=str)
def test_a_plan_of_another_configuration_is_refused_for_that(other):
    made = dict(T=4, k=2, E=3, d=16, dtype=etr.BF16)
    plan = etr.SortBuffers(etr.make_sort_config(**made), device="cpu")
    cfg = etr.make_sort_config(**dict(made, **other))
    for name, call in sort_calls(plan.cfg, plan).items():
        refused(lambda: call(cfg), etr.ERR_WORKSPACE, name, "plan: made for another configuration")


def test_a_plan_keeps_the_configuration_that_it_was_made_for():
    """Whatever becomes of the two configurations that a caller can reach, its own and the plan's."""
    cfg = etr.make_sort_config(T=4, k=2, E=3, d=16, dtype=etr.BF16)
    plan = etr.SortBuffers(cfg, device="cpu")
    assert bytes(plan.cfg) == bytes(cfg)
    cfg.T = plan.cfg.T = 5
    for name, call in sort_calls(cfg, plan).items():
        refused(lambda: call(plan.cfg), etr.ERR_WORKSPACE, name, "plan: made for another configuration")


# ---- the composed calls ------------------------------------------------------------------------------
LAYER = dict(T=4, d=64, D=8, E=4, k=2, h=64, capacity=4, dtype=etr.BF16)


def composed_calls(buf, plan, bb):
    """Every composed call under a given configuration, its tensors left out."""
    return {"etr_routed_forward": lambda c, n: etr.routed_forward(c, *[None] * 6, buf, plan, None),
            "etr_routed_backward": lambda c, n: etr.routed_backward(c, *[None] * 5, buf, plan, *[None] * 5),
            "etr_block_forward": lambda c, n: etr.block_forward(c, n, *[None] * 8, buf, bb, None),
            "etr_block_backward": lambda c, n: etr.block_backward(c, n, *[None] * 9, buf, bb, *[None] * 8)}


def made(**kw):
    cfg, device = etr.make_config(**dict(LAYER, **kw)), "cpu"
    n = etr.make_norm_config(T=cfg.T, d=cfg.d, dtype=cfg.dtype)
    return cfg, n, etr.LayerBuffers(cfg, device=device), etr.SortBuffers(etr.routed_sort_config(cfg), device=device), etr.BlockBuffers(n, device=device)


def test_composed_calls_refuse_buffers_that_are_not_on_a_gpu():
    cfg, n, buf, plan, bb = made()
    for name, call in composed_calls(buf, plan, bb).items():
        refused(lambda: call(cfg, n), etr.ERR_ARG, name, "buf: not on a CUDA device")
        buf._for.device = 0                                  # the other handle is looked at as well
        refused(lambda: call(cfg, n), etr.ERR_ARG, name, "plan: " if "routed" in name else "bb: ", "not on a CUDA device")
        buf._for.device = -1


@pytest.mark.parametrize("other", [dict(T=5), dict(k=1), dict(E=3), dict(capacity=200)], ids=str)
def test_composed_calls_refuse_a_plan_of_another_configuration(other):
    cfg, n, buf, _, bb = made()
    plan = etr.SortBuffers(etr.routed_sort_config(etr.make_config(**dict(LAYER, **other))), device="cpu")
    for name, call in composed_calls(buf, plan, bb).items():
        if "routed" in name:
            refused(lambda: call(cfg, n), etr.ERR_WORKSPACE, name, "plan: made for another configuration")


@pytest.mark.parametrize("other, experts, router", [
    # members as long as the batch: the layer's own router's alone
    (dict(T=3), True, False), (dict(k=1), True, False), (dict(D=16), True, False), (dict(E=2, capacity=200), True, False),
    (dict(E=3), False, False), (dict(d=32, D=4), False, False), (dict(h=32), False, False), (dict(capacity=0x80, E=3), False, False),
    (dict(T=5, E=5, k=3, d=128, h=128, capacity=300), True, True), (dict(dtype=etr.F32), True, True), (dict(), True, True)], ids=str)
def test_composed_calls_refuse_buffers_of_a_smaller_layer(other, experts, router):
    """Buffers of a larger one serve as they do for the layer's own calls: what is wrong then is that these are not on a GPU."""
    small = etr.LayerBuffers(etr.make_config(**dict(LAYER, gemm_impl=etr.GEMM_SIMT, **other)), device="cpu")
    cfg, n, _, plan, bb = made()
    for name, call in composed_calls(small, plan, bb).items():
        if router if "block" in name else experts:
            refused(lambda: call(cfg, n), etr.ERR_ARG, name, "buf: not on a CUDA device")
        else:
            refused(lambda: call(cfg, n), etr.ERR_WORKSPACE, name, "buf: made for another configuration")


@pytest.mark.parametrize("other", [dict(T=5), dict(d=128), dict(dtype=etr.F32)], ids=str)
def test_composed_calls_refuse_block_buffers_of_another_configuration(other):
    cfg, n, buf, plan, _ = made()
    bb = etr.BlockBuffers(etr.make_norm_config(**dict(dict(T=4, d=64, dtype=etr.BF16), **other)), device="cpu")
    for name, call in composed_calls(buf, plan, bb).items():
        if "block" in name:
            refused(lambda: call(cfg, n), etr.ERR_WORKSPACE, name, "bb: made for another configuration")


def test_composed_calls_check_the_configuration_first():
    cfg, n, buf, plan, bb = made()
    for bad, code in ((dict(k=5), etr.ERR_SHAPE), (dict(h=0), etr.ERR_ARG), (dict(D=0), etr.ERR_ARG)):
        for name, call in composed_calls(buf, plan, bb).items():
            refused(lambda: call(etr.make_config(**dict(LAYER, **bad)), n), code, name)


ROUTE = ("topk_idx", "counts", "slot_token", "gate", "tok_ptr", "tok_row")
FORWARD = ("G", "U", "H", "O", "ws")
BACKWARD = ("dO", "dG", "dU", "dXp")


def changed(struct, name, value):
    s = type(struct).from_buffer_copy(struct)
    setattr(s.route if isinstance(s, etr.Buffers) and name in ROUTE else s, name, value)
    return C.byref(s)


@pytest.mark.parametrize("kw", [dict(), dict(gate_mode=etr.GATE_SOFTMAX), dict(fuse_dispatch=etr.FUSE_ON), dict(weight_dtype=etr.F32),
                                dict(k=1), dict(dtype=etr.F32)], ids=str)
def test_composed_calls_check_every_member_before_anything_runs(kw):
    """A block's call launches the norm before the layer looks at its buffers, and the routed call clears the stats before the
    plan is looked at: both have to know first."""
    cfg = etr.make_config(**dict(dict(T=64, d=256, D=8, E=8, k=2, h=128, capacity=64, dtype=etr.BF16), **kw))
    names, call, buf = composed(cfg, etr.make_norm_config(T=64, d=256, dtype=cfg.dtype, post_norm=True))
    ok, soft, tensor_cores = 1 << 20, cfg.gate_mode == etr.GATE_SOFTMAX, cfg.dtype == etr.BF16
    xp = () if cfg.fuse_dispatch == etr.FUSE_ON else ("Xp",)
    affinity = ("delta", "xnorm", "rnorm") + (("lse",) if soft else ())
    need = {"etr_routed_forward": FORWARD + ("Xp", "stats"), "etr_routed_backward": FORWARD + BACKWARD + ("Xp", "stats"),
            "etr_block_forward": FORWARD + xp + affinity + ROUTE + ("stats",),
            "etr_block_backward": FORWARD + BACKWARD + xp + affinity + ROUTE + ("dgate",) + (("ddelta",) if soft else ()) +
            (("stats",) if tensor_cores else ())}
    for name in names:
        for x in need[name]:
            for value, code in ((None, etr.ERR_ARG), (ok + 4, etr.ERR_ALIGN)):
                assert call(name, buf=changed(buf, x, value)) == code, (name, x)
        if "routed" in name:
            for x, _ in etr.SortPlan._fields_:
                for value, code in ((None, etr.ERR_ARG), (ok + 4, etr.ERR_ALIGN)):
                    assert call(name, plan=changed(etr.SortPlan(*[ok] * 6), x, value)) == code, (name, x)
    assert call("etr_block_forward", buf=changed(buf, "Z", ok + 4)) == etr.ERR_ALIGN
    assert call("etr_block_backward", buf=changed(buf, "Z", None)) == etr.ERR_ARG
