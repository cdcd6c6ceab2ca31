"""Calls of the row operators that the Python binding refuses before it reaches the library, without a GPU."""
import pytest
import torch

from paper_2406_00023_b200 import etr


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
    layer = etr.make_config(T=4, d=64, D=8, E=4, k=2, h=64, capacity=4, dtype=etr.BF16)
    plan, buf = etr.SortBuffers(etr.routed_sort_config(layer), device="cpu"), etr.LayerBuffers(layer, device="cpu")
    refused(lambda: etr.routed_forward(layer, None, None, None, None, None, None, buf, plan, None), etr.ERR_ARG, "plan: not on a CUDA device")
    refused(lambda: etr.routed_backward(layer, None, None, None, None, None, buf, plan, None, None, None, None, None), etr.ERR_ARG,
            "plan: not on a CUDA device")


@pytest.mark.parametrize("other", [dict(T=5), dict(k=1), dict(E=4), dict(align=2), dict(align=128, capacity=4)], ids=str)
def test_a_plan_of_another_configuration_is_refused_for_that(other):
    made = dict(T=4, k=2, E=3, d=16, dtype=etr.BF16)
    plan = etr.SortBuffers(etr.make_sort_config(**made), device="cpu")
    cfg = etr.make_sort_config(**dict(made, **other))
    for name, call in sort_calls(plan.cfg, plan).items():
        refused(lambda: call(cfg), etr.ERR_WORKSPACE, name, "plan: made for another configuration")
