"""Tokens sorted by a given choice of experts and back, on the GPU: the plan number for number, the row passes against their
64-bit definitions (tests/rows_reference.py has the bounds)."""
import pytest
import torch

from paper_2406_00023_b200 import etr
from tests import rows_reference as rr

pytestmark = pytest.mark.gpu
DT = {torch.bfloat16: etr.BF16, torch.float32: etr.F32}
UNTOUCHED = -12345


def make(T, k, E, d, dtype=torch.bfloat16, align=1, capacity=0):
    cfg = etr.make_sort_config(T=T, k=k, E=E, d=d, dtype=DT[dtype], align=align, capacity=capacity)
    buf = etr.SortBuffers(cfg)
    buf.block.fill_(0x5a)
    return cfg, buf


def choice(T, k, E, seed, lost=0.2):
    """Ids of all kinds: in range, skewed, repeated within a token, out of range on both sides."""
    g = torch.Generator().manual_seed(seed)
    ids = (torch.rand(T, k, generator=g) ** 2 * E).long().clamp(max=E - 1)
    wrong = torch.tensor([-1, E, E + 7, -(1 << 31), (1 << 31) - 1])
    out = torch.rand(T, k, generator=g) < lost
    return torch.where(out, wrong[torch.randint(0, 5, (T, k), generator=g)], ids).to(torch.int32)


def check_plan(cfg, buf, ids):
    want = rr.plan(ids, cfg.E, cfg.align, cfg.capacity, buf.n_rows)
    for name, w in zip(("counts", "offsets", "totals", "row_token", "pos"), want):
        assert getattr(buf, name).cpu().tolist() == w, name


SHAPES = [(0, 2, 3), (1, 1, 1), (1, 8, 16), (2, 3, 1000), (31, 1, 2), (33, 2, 16), (64, 2, 16), (129, 8, 128), (511, 32, 7), (513, 2, 16),
          (1024, 1, 1), (2050, 3, 12), (5000, 8, 1024), (8193, 4, 33)]


@pytest.mark.parametrize("T, k, E", SHAPES)
@pytest.mark.parametrize("form", [(1, 0), (8, 0), (1000, 0), (128, "even"), (128, 1), (128, "all")], ids=str)
def test_plan(T, k, E, form):
    align, capacity = form
    capacity = {"even": max(1, T * k // E), "all": max(1, T)}.get(capacity, capacity)
    cfg, buf = make(T, k, E, 8, align=align, capacity=capacity)
    for seed in (1, 2):                                    # the second choice finds the first one's plan in the buffers
        ids = choice(T, k, E, seed)
        etr.sort(cfg, ids.cuda(), buf)
        check_plan(cfg, buf, ids)


@pytest.mark.parametrize("ids", [torch.full((300, 2), -1), torch.full((300, 2), 5), torch.zeros(300, 2), torch.full((300, 2), 15)],
                         ids=["nobody", "one", "first", "last"])
@pytest.mark.parametrize("capacity", [0, 100])
def test_plan_of_one_sided_choices(ids, capacity):
    cfg, buf = make(300, 2, 16, 8, align=128 if capacity else 4, capacity=capacity)
    ids = ids.to(torch.int32)
    etr.sort(cfg, ids.cuda(), buf)
    check_plan(cfg, buf, ids)


@pytest.mark.parametrize("T, k, E, skew", [(65536, 2, 64, 1), (65536, 8, 256, 1), (70001, 5, 1000, 3), (300000, 1, 3, 1)])
def test_plan_of_long_batches(T, k, E, skew):
    """Against a stable sort."""
    g = torch.Generator().manual_seed(T)
    ids = (torch.rand(T, k, generator=g) ** skew * E).int().clamp(max=E - 1)
    cfg, buf = make(T, k, E, 8)
    etr.sort(cfg, ids.cuda(), buf)
    flat = ids.reshape(-1).long()
    order = torch.sort(flat, stable=True).indices
    assert torch.equal(buf.counts.cpu().long(), torch.bincount(flat, minlength=E))
    assert torch.equal(buf.row_token.cpu().long(), order // k)
    assert torch.equal(buf.pos.cpu().long().reshape(-1)[order], torch.arange(T * k))
    assert buf.totals.cpu().tolist() == [T * k, 0, 0, 0]


ROWS = [(0, 2, 3, 16), (1, 1, 1, 8), (1, 8, 16, 64), (7, 3, 5, 72), (64, 2, 16, 1024), (129, 8, 128, 264), (300, 32, 7, 8),
        (513, 2, 16, 4096), (100, 3, 12, 1088), (50, 4, 9, 8200),
        # more pairs than the walking blocks of the weights' gradient have warps, more pieces than one round of every SM's threads
        (2000, 3, 16, 512), (20000, 4, 16, 64), (3000, 1, 5, 2048), (40000, 1, 700, 136),
        (3000, 2, 5, 2048), (3001, 3, 5, 2056), (5000, 4, 9, 1088)]


@pytest.mark.parametrize("T, k, E, d", ROWS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("form", [(1, 0), (16, 0), (128, "cut")], ids=str)
def test_rows_and_their_gradients(T, k, E, d, dtype, form):
    align, capacity = form
    capacity = max(1, T * k // E // 2) if capacity == "cut" else 0
    cfg, buf = make(T, k, E, d, dtype, align, capacity)
    ids = choice(T, k, E, 3 * T + k)
    etr.sort(cfg, ids.cuda(), buf)
    g = torch.Generator(device="cuda").manual_seed(d)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dtype)                           # noqa: E731
    R, pos, pick = buf.n_rows, buf.pos, buf.pos >= 0
    token_rows, pad = buf.row_token >= 0, torch.zeros(R, dtype=torch.bool, device="cuda")
    for o, c in zip(buf.offsets.cpu().tolist(), buf.counts.cpu().tolist()):
        pad[o + c:o + -(-c // align) * align] = True
    X, dY = rand(T, d), rand(T, d)
    w = torch.rand(T, k, generator=g, device="cuda") - 0.3
    w[~pick] = float("nan")                                # weights without a row are not read
    O, dXs = rand(R, d), rand(R, d)
    O[~token_rows] = float("nan")                          # neither are rows without a token
    dXs[~token_rows] = float("nan")
    Xs, dO = (torch.full((R, d), UNTOUCHED, dtype=dtype, device="cuda") for _ in range(2))
    Y, dX = (torch.full((T, d), UNTOUCHED, dtype=dtype, device="cuda") for _ in range(2))
    dw = torch.full((T, k), float("nan"), device="cuda")
    etr.sort_rows(cfg, X, buf, Xs)
    etr.unsort_rows(cfg, O, w, buf, Y)
    etr.unsort_rows_bwd(cfg, dY, O, w, buf, dO, dw)
    etr.sort_rows_bwd(cfg, dXs, buf, dX)
    torch.cuda.synchronize()
    want = torch.full((R, d), UNTOUCHED, dtype=dtype, device="cuda")
    want[pad] = 0
    want[token_rows] = X[buf.row_token[token_rows].long()]
    assert torch.equal(Xs, want)                           # rows behind the pad rows are as they were
    rr.assert_within(Y, *rr.unsort(O, w, pos, dtype), "Y")
    rr.assert_within(dX, *rr.unsort(dXs, None, pos, dtype), "dX")
    (ref, bound), (dw_ref, dw_bound) = rr.unsort_bwd(dY, O, w, pos, R, dtype)
    rr.assert_within(dO[token_rows], ref[token_rows], bound[token_rows], "dO")
    assert bool((dO[pad] == 0).all()) and bool((dO[~token_rows & ~pad] == UNTOUCHED).all())
    rr.assert_within(dw, dw_ref, dw_bound, "dweights")
    assert bool((dw[~pick] == 0).all())


def test_special_values_stay_in_their_token():
    T, k, E, d = 40, 2, 4, 64
    cfg, buf = make(T, k, E, d)
    ids = choice(T, k, E, 5, lost=0.0)
    etr.sort(cfg, ids.cuda(), buf)
    O = torch.randn(buf.n_rows, d, device="cuda").bfloat16()
    w = torch.rand(T, k, device="cuda")
    Y, clean = torch.empty(T, d, dtype=torch.bfloat16, device="cuda"), torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    etr.unsort_rows(cfg, O, w, buf, clean)
    O[buf.pos[3, 0].long(), 5] = float("nan")
    O[buf.pos[7, 1].long(), 6] = float("inf")
    etr.unsort_rows(cfg, O, w, buf, Y)
    other = torch.ones(T, d, dtype=torch.bool, device="cuda")
    other[3, 5] = other[7, 6] = False
    assert torch.equal(Y[other], clean[other]) and bool(Y[3, 5].isnan()) and bool(Y[7, 6].isinf())


def test_same_bits_every_time_and_on_another_stream():
    T, k, E, d = 3001, 3, 12, 1088
    cfg, buf = make(T, k, E, d)
    ids = choice(T, k, E, 9).cuda()
    X, w = torch.randn(T, d, device="cuda").bfloat16(), torch.rand(T, k, device="cuda")
    outs = []
    side = torch.cuda.Stream()
    for stream in (torch.cuda.current_stream(), side, side):
        Xs, dO = torch.zeros(buf.n_rows, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(buf.n_rows, d, dtype=torch.bfloat16, device="cuda")
        Y, dw = torch.empty(T, d, dtype=torch.bfloat16, device="cuda"), torch.empty(T, k, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            etr.sort(cfg, ids, buf)
            etr.sort_rows(cfg, X, buf, Xs)
            etr.unsort_rows(cfg, Xs, w, buf, Y)
            etr.unsort_rows_bwd(cfg, X, Xs, w, buf, dO, dw)
        torch.cuda.synchronize()
        outs.append([t.clone() for t in (Xs, Y, dO, dw, buf.pos)])
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))


def test_captured_calls_follow_the_choice():
    T, k, E, d = 700, 2, 16, 256
    cfg, buf = make(T, k, E, d, align=16)
    ids, X, w = choice(T, k, E, 1).cuda(), torch.randn(T, d, device="cuda").bfloat16(), torch.rand(T, k, device="cuda")
    Xs, Y = torch.zeros(buf.n_rows, d, dtype=torch.bfloat16, device="cuda"), torch.empty(T, d, dtype=torch.bfloat16, device="cuda")

    def calls():
        etr.sort(cfg, ids, buf)
        etr.sort_rows(cfg, X, buf, Xs)
        etr.unsort_rows(cfg, Xs, w, buf, Y)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed in (2, 3):
        now = choice(T, k, E, seed)
        ids.copy_(now)
        w.uniform_()
        graph.replay()
        torch.cuda.synchronize()
        check_plan(cfg, buf, now)
        rr.assert_within(Y, *rr.unsort(Xs, w, buf.pos, torch.bfloat16), "Y")


def test_rows_beyond_32_bit_offsets():
    """Buffers of more than 2^31 elements: the last rows as well as the first."""
    T, k, E, d = 70000, 2, 2, 16384
    cfg, buf = make(T, k, E, d)
    ids = torch.tensor([0, 1], dtype=torch.int32, device="cuda").repeat(T, 1).contiguous()
    etr.sort(cfg, ids, buf)
    X = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    X.copy_((torch.arange(T, device="cuda") % 251).bfloat16()[:, None].expand(T, d))
    Xs = torch.zeros(2 * T, d, dtype=torch.bfloat16, device="cuda")
    etr.sort_rows(cfg, X, buf, Xs)
    assert torch.equal(Xs[:T], X) and torch.equal(Xs[T:], X)
    Y, w = torch.empty_like(X), torch.full((T, k), 0.5, device="cuda")
    etr.unsort_rows(cfg, Xs, w, buf, Y)
    assert torch.equal(Y, X)
    dO, dw = torch.zeros_like(Xs), torch.empty(T, k, device="cuda")
    etr.unsort_rows_bwd(cfg, X, Xs, w, buf, dO, dw)
    assert torch.equal(dO[T:], X / 2)
    # partial sums are m v^2 with v^2 below 2^16 and m up to d = 2^14: up to 30 bits, so not all of them fp32 numbers
    ref = ((torch.arange(T, device="cuda") % 251).double().square() * d)[:, None].expand(T, k)
    rr.assert_within(dw, ref, (d + 1) * rr.U * ref, "dweights")
    etr.sort_rows_bwd(cfg, Xs, buf, Y)
    assert torch.equal(Y, X * 2)


def test_calls_are_refused_before_a_launch():
    cfg, buf = make(10, 2, 4, 64)
    X, Xs = torch.zeros(10, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(20, 64, dtype=torch.bfloat16, device="cuda")
    n0 = etr.launch_count()
    for bad, code in ((X.float(), etr.ERR_ARG), (X[:9], etr.ERR_SHAPE), (X.cpu(), etr.ERR_ARG), (X.t(), etr.ERR_SHAPE), (None, etr.ERR_ARG),
                      (torch.zeros(641, dtype=torch.bfloat16, device="cuda")[1:], etr.ERR_ALIGN)):
        with pytest.raises(etr.EtrError) as e:
            etr.sort_rows(cfg, bad, buf, Xs)
        assert e.value.code == code
    with pytest.raises(etr.EtrError) as e:
        etr.sort(cfg, torch.zeros(10, 2, dtype=torch.int64, device="cuda"), buf)
    assert e.value.code == etr.ERR_ARG
    for other in (dict(T=9), dict(k=3), dict(E=5), dict(align=8), dict(align=128, capacity=8)):       # a plan of another configuration
        c = etr.make_sort_config(**dict(dict(T=10, k=2, E=4, d=64, dtype=etr.BF16), **other))
        with pytest.raises(etr.EtrError) as e:
            etr.sort(c, torch.zeros(c.T, c.k, dtype=torch.int32, device="cuda"), buf)
        assert e.value.code == etr.ERR_WORKSPACE
    cfg.T = 11                                             # the buffers keep the configuration they were made for
    with pytest.raises(etr.EtrError) as e:
        etr.sort(cfg, torch.zeros(11, 2, dtype=torch.int32, device="cuda"), buf)
    assert e.value.code == etr.ERR_WORKSPACE
    assert etr.launch_count() == n0
