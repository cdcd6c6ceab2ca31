"""The plan of choices of more pairs than one cluster takes: a counting launch, prefix sums across clusters, gaps filled by all
warps.  Every array against a stable sort, two choices on the same buffers."""
import pytest
import torch

from paper_2406_00023_b200 import etr
from tests import rows_reference as rr

pytestmark = pytest.mark.gpu


def sorted_plan(ids, E, align, capacity, n_rows):
    """counts, offsets, totals, row_token, pos by one stable sort of the pairs."""
    T, k = ids.shape
    flat = ids.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < E), flat, E)
    found = torch.bincount(key, minlength=E + 1)[:E]
    counts = found.clamp(max=capacity) if capacity else found
    rows = torch.full_like(counts, -(-capacity // 128) * 128) if capacity else -(-counts // align) * align
    offsets = torch.zeros(E + 1, dtype=torch.long)
    offsets[1:] = rows.cumsum(0)
    order = torch.sort(key, stable=True).indices
    first = torch.zeros(E + 1, dtype=torch.long)
    first[1:] = found.cumsum(0)
    rank = torch.arange(T * k) - first[key[order]]
    kept = rank < torch.cat([counts, torch.zeros(1, dtype=torch.long)])[key[order]]
    row = torch.where(kept, offsets[key[order]] + rank, -1)
    pos, row_token = torch.empty(T * k, dtype=torch.long), torch.full((n_rows,), -1)
    pos[order] = row
    row_token[row[kept]] = (order // k)[kept]
    with_row, with_expert = int(counts.sum()), int(found.sum())
    return counts, offsets, torch.tensor([with_row, with_expert - with_row, T * k - with_expert, 0]), row_token, pos.view(T, k)


def choice(T, k, E, seed, lost, skew):
    g = torch.Generator().manual_seed(seed)
    ids = (torch.rand(T, k, generator=g, dtype=torch.float64) ** skew * E).long().clamp(max=E - 1)
    wrong = torch.tensor([-1, E, E + 7, -(1 << 31), (1 << 31) - 1])
    out = torch.rand(T, k, generator=g) < lost
    return torch.where(out, wrong[torch.randint(0, 5, (T, k), generator=g)], ids).to(torch.int32)


def check(cfg, buf, ids):
    for name, want in zip(("counts", "offsets", "totals", "row_token", "pos"), sorted_plan(ids, cfg.E, cfg.align, cfg.capacity, buf.n_rows)):
        got = getattr(buf, name).cpu().long()
        assert torch.equal(got, want), (name, int((got != want).sum()))


def test_the_sorted_plan_is_the_plan_by_hand():
    """The reference of these tests against the one that goes pair by pair."""
    for T, k, E, align, capacity in ((50, 3, 7, 1, 0), (50, 3, 7, 16, 0), (50, 3, 7, 128, 9)):
        ids = choice(T, k, E, T, 0.2, 2.0)
        n = etr.sort_n_rows(etr.make_sort_config(T=T, k=k, E=E, d=8, dtype=etr.F32, align=align, capacity=capacity))
        assert [x.tolist() for x in sorted_plan(ids, E, align, capacity, n)] == list(rr.plan(ids, E, align, capacity, n))


FORMS = [(1, None), (8, None), (128, None), (1000, None), (128, "half"), (128, "even"), (128, "all")]


@pytest.mark.parametrize("T, k, E", [(65537, 1, 64), (32769, 2, 3), (9001, 8, 1024), (70001, 5, 1000), (50000, 12, 40), (150001, 1, 1)])
@pytest.mark.parametrize("align, share", FORMS, ids=str)
def test_plan_across_clusters(T, k, E, align, share):
    capacity = {None: 0, "half": max(1, T * k // E // 2), "even": max(1, T * k // E), "all": T * k if E == 1 else T * k // 2}[share]
    if capacity and E * capacity > 1 << 24:
        capacity = (1 << 24) // E
    cfg = etr.make_sort_config(T=T, k=k, E=E, d=8, dtype=etr.BF16, align=align, capacity=capacity)
    buf = etr.SortBuffers(cfg)
    buf.block.fill_(0x5a)
    for seed, lost, skew in ((1, 0.15, 1.0), (2, 0.0, 4.0)):           # the second finds the first one's plan and counts in the buffers
        ids = choice(T, k, E, seed, lost, skew)
        etr.sort(cfg, ids.cuda(), buf)
        check(cfg, buf, ids)


@pytest.mark.parametrize("ids", [-1, 0, 16, 31, 40], ids=["nobody", "first", "one", "last", "out_of_range"])
@pytest.mark.parametrize("align, capacity", [(1, 0), (4, 0), (128, 100), (128, 99999)], ids=str)
def test_one_sided_choices_across_clusters(ids, align, capacity):
    T, k, E = 33333, 3, 32
    cfg = etr.make_sort_config(T=T, k=k, E=E, d=8, dtype=etr.BF16, align=align, capacity=capacity)
    buf = etr.SortBuffers(cfg)
    buf.block.fill_(0x5a)
    etr.sort(cfg, choice(T, k, E, 3, 0.5, 1.0).cuda(), buf)
    ids = torch.full((T, k), ids, dtype=torch.int32)
    etr.sort(cfg, ids.cuda(), buf)
    check(cfg, buf, ids)


def test_rows_across_clusters():
    """The passes on such a plan, with gaps, drops and lost choices: the rows and both ways back."""
    T, k, E, d = 40000, 3, 24, 64
    for align, capacity in ((16, 0), (128, 3000)):
        cfg = etr.make_sort_config(T=T, k=k, E=E, d=d, dtype=etr.BF16, align=align, capacity=capacity)
        buf = etr.SortBuffers(cfg)
        ids = choice(T, k, E, 5, 0.1, 2.0)
        etr.sort(cfg, ids.cuda(), buf)
        check(cfg, buf, ids)
        X, w = torch.randn(T, d, device="cuda").bfloat16(), torch.rand(T, k, device="cuda")
        Xs, Y, dX = torch.full((buf.n_rows, d), 7.0, device="cuda").bfloat16(), torch.empty_like(X), torch.empty_like(X)
        etr.sort_rows(cfg, X, buf, Xs)
        live = buf.row_token >= 0
        assert torch.equal(Xs[live], X[buf.row_token[live].long()])
        etr.unsort_rows(cfg, Xs, w, buf, Y)
        etr.sort_rows_bwd(cfg, Xs, buf, dX)
        rr.assert_within(Y, *rr.unsort(Xs, w, buf.pos, X.dtype), "Y")
        rr.assert_within(dX, *rr.unsort(Xs, None, buf.pos, X.dtype), "dX")


@pytest.mark.parametrize("lost", [0, 300])
def test_the_most_pairs_that_a_plan_takes(lost):
    """2^31 - 65537 pairs, pair i of expert i mod 7, the last `lost` without an expert: the rows are known without a sort.  Behind the
    last row nothing, or 300 rows without a token, are left to fill."""
    n, E, step = 2 ** 31 - 65537, 7, 1 << 28
    cfg = etr.make_sort_config(T=n, k=1, E=E, d=8, dtype=etr.BF16)
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("60 GB of device memory")
    buf = etr.SortBuffers(cfg)
    ids = torch.empty(n, 1, dtype=torch.int32, device="cuda")
    for i in range(0, n, step):
        ids[i:i + step, 0] = torch.arange(i, min(i + step, n), device="cuda") % E
    ids[n - lost:] = -1
    etr.sort(cfg, ids, buf)
    del ids
    kept = n - lost
    counts = torch.tensor([(kept + E - 1 - e) // E for e in range(E)])
    offsets = torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)])
    assert buf.counts.tolist() == counts.tolist() and buf.offsets.tolist() == offsets.tolist() and buf.totals.tolist() == [kept, 0, lost, 0]
    start = offsets.cuda()
    for i in range(0, n, step):
        at = torch.arange(i, min(i + step, n), device="cuda")
        row = torch.where(at < kept, start[at % E] + at // E, -1)
        assert torch.equal(buf.pos[i:i + step, 0].long(), row)
        has = row >= 0
        assert torch.equal(buf.row_token[row[has]].long(), at[has])
    assert bool((buf.row_token[kept:] == -1).all())
