"""Answers where sums are long, rows have no finite logit, single table rows are far larger than the rest, and rows go in turns."""
import math

import pytest
import torch

from tests import dense_util as du
from tests import layers_util as lu
from tests.dense_util import E

pytestmark = pytest.mark.gpu

# The sums of the exponentials: of 16 in a lane (15 E), times one factor (4 E), added up in 64 bits whatever the table's length; the joins of
# waves, splits and lanes, 24 at most, are an E each besides the exponentials that bring them to one maximum (2 E each).  With the
# exponential's and the logarithm's own error: 128 E.
SUM = 128 * E


@pytest.fixture(scope="module")
def recd():
    from paper_2211_05239_amd import recd as mod
    return mod


@pytest.fixture(scope="module")
def ctx(recd):
    c = recd.Context(0)
    yield c
    c.close()


def answers(ctx, x, table, scale=1.0, k=0):
    n = len(x)
    lse, entropy = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ids, logs = (torch.empty(n, k, dtype=torch.int64, device="cuda"), torch.empty(n, k, device="cuda")) if k else (None, None)
    ctx.vocab_answers(x, table, scale, entropy=entropy, lse=lse, top_ids=ids, top_logp=logs)
    return lse, entropy, ids, logs


# by the kernel of many rows in one split, in a few, and by that of few rows
@pytest.mark.parametrize("n,V,k", [(131_072, 1_000_001, 0), (9000, 1_000_001, 2), (300, 1_000_001, 2), (3, 4_000_001, 2)])
def test_one_large_logit_over_many_equal_ones(ctx, n, V, k):
    """Adding the same small value over and over rounds the same way each time.  One row of the table has the logit a, all others b, with
    (V - 1) exp(b - a) from 2^-6 to 2^6; in 64 bits: lse = a + log1p((V - 1) exp(b - a)).  Products and sums of the logits are exact: a is a multiple of 2^-3, b 0."""
    table = torch.zeros(V, 8, dtype=torch.bfloat16, device="cuda")
    table[:, 1] = 1.0
    table[V // 3, 1] = 0.0
    table[V // 3, 0] = 1.0
    x = torch.zeros(n, 8, dtype=torch.bfloat16, device="cuda")
    gap = math.log(V) + (torch.arange(n, device="cuda") % 97 - 48) * math.log(2.0) / 8
    x[:, 0] = (gap.double() * 8).round().bfloat16() / 8
    lse, entropy, ids, logs = answers(ctx, x, table, 1.0, k)
    a = x[:, 0].double()
    q = (V - 1) * torch.exp(-a)                                                       # b = 0
    want = a + torch.log1p(q)
    p0, rest = 1 / (1 + q), q / (1 + q)
    H = p0 * torch.log1p(q) + rest * want
    # a logit in powers of two, less the maximum, is off by three roundings of up to 1.45 a
    dz = 8 * E * a
    assert ((lse.double() - want).abs() <= dz + SUM + E * want.abs()).all(), float((lse.double() - want).abs().max())
    assert ((entropy.double() - H).abs() <= dz * (1 + H) + SUM * (1 + H) + 4 * E * (1 + H) * want).all(), float((entropy.double() - H).abs().max())
    if k:
        other = 0 if V // 3 else 1
        assert (ids[:, 0] == V // 3).all() and (ids[:, 1] == other).all()
        assert ((logs[:, 1].double() + want).abs() <= dz + SUM + E * want.abs()).all()


@pytest.mark.parametrize("dt,n,V,D", [("bf16", 70_000, 30_011, 16), ("f32", 70_000, 10_001, 8), ("f16", 300, 200_003, 16), ("f32", 3, 1_000_003, 16)])
def test_sums_do_not_lose_with_the_table(ctx, dt, n, V, D):
    """Against 64 bits, with a bound of the sums that does not grow with V."""
    x, table = du.rand((n, D), dt, 1), du.rand((V, D), dt, 2, 2.0 / D ** 0.5)
    lse, entropy, _, _ = answers(ctx, x.cuda(), table.cuda())
    rows = torch.randperm(n, generator=torch.Generator().manual_seed(3))[:20]
    x = x[rows]
    z = x.double() @ table.double().t()
    size = x.double().abs() @ table.double().abs().t()
    want = torch.logsumexp(z, 1)
    p = (z - want[:, None]).exp()
    H = torch.special.entr(p).sum(1)
    dz = 4 * E * (D + 8) * size + 8 * E * (z.abs() + want.abs()[:, None])
    assert ((lse.cpu()[rows].double() - want).abs() <= (p * dz).sum(1) + SUM + 2 * E * want.abs()).all()
    dH = ((p * (z - want[:, None] + H[:, None]).abs()) * dz).sum(1)
    assert ((entropy.cpu()[rows].double() - H).abs() <= dH + SUM * (1 + H) + 2 * E * H).all()


@pytest.mark.parametrize("n", [3, 300])
@pytest.mark.parametrize("size", [1e4, 1e7, 1e10, 1e15, 1e25])
def test_large_logits(ctx, n, size):
    """The difference of a score and the running maximum has digits that the maximum itself is rounded off."""
    g = torch.Generator().manual_seed(4)
    x, table = torch.rand(n, 4, generator=g) + 0.5, torch.rand(700, 4, generator=g) - 0.5
    for order in (1, -1):
        rows = table[(table.sum(1) * order).argsort()] * size        # the maximum rises all along, or comes first
        lse, entropy, ids, _ = answers(ctx, x.cuda(), rows.cuda(), 1.0, 3)
        z = x.double() @ rows.double().t()
        want = torch.logsumexp(z, 1)
        p = (z - want[:, None]).exp()
        dz = 4 * E * 12 * (x.double() @ rows.double().abs().t()) + 8 * E * (z.abs() + want.abs()[:, None])
        assert lse.isfinite().all() and entropy.isfinite().all()
        # a logit is off by far more than 1 from 1e10 on: what the others can add to the largest is log(700) at most
        assert ((lse.double().cpu() - want).abs() <= dz.max(1).values + SUM + E * want.abs()).all()
        assert (entropy >= 0).all() and (entropy <= math.log(700) + 1e-3).all()
        assert torch.equal(ids.cpu(), z.sort(dim=1, descending=True, stable=True)[1][:, :3])


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [3, 300])
@pytest.mark.parametrize("V", [1, 31, 64, 65, 200, 4097])
def test_rows_with_no_finite_logit(ctx, dt, n, V):
    """-infinity everywhere: so is lse, what stands behind the table's last row is no logit, and of equal ones the lowest ids come first."""
    x, table = du.rand((n, 16), dt, 1), du.rand((V, 16), dt, 2).abs()
    table[:, 0] = 1.0
    x[1] = 0.0
    x[1, 0] = -math.inf
    k = min(V, 5)
    lse, _, ids, _ = answers(ctx, x.cuda(), table.cuda(), 1.0, k)
    assert lse[1].item() == -math.inf and torch.equal(ids[1].cpu(), torch.arange(k))
    rest = [i for i in range(n) if i != 1]
    z = lu.logits(x[rest[:20]], table, 1.0)
    assert torch.equal(ids.cpu()[rest[:20]], z.sort(dim=1, descending=True, stable=True)[1][:, :k])
    assert lse[rest].isfinite().all()


def test_logits_below_the_places_behind_the_table(ctx):
    """Finite logits near the end of the range, in a table that ends inside a tile."""
    for V in (1, 3, 33, 70):
        for a in (-5e37, -1.2e38, -2e38):
            table = torch.zeros(V, 4)
            table[:, 0] = 1.0
            x = torch.zeros(300, 4)
            x[:, 0] = a
            for m in (3, 300):
                lse, _, _, _ = answers(ctx, x[:m].cuda(), table.cuda())
                assert ((lse.double().cpu() - (x[:m, 0].double() + math.log(V))).abs() <= 4 * E * abs(a)).all(), (V, a)


# an outlier in the table: in its first, a middle and its last row (that of a part of a chunk)
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [3, 300])
@pytest.mark.parametrize("at,by", [(0, 1e4), (7777, -1e4), (20_000, 300.0)])
def test_one_row_of_large_values(ctx, dt, n, at, by):
    x, table = du.rand((n, 64), dt, 1), du.rand((20_001, 64), dt, 2, 0.2)
    table[at, 5] = by
    lse, entropy, ids, logs = answers(ctx, x.cuda(), table.cuda(), 1.0, 9)
    some = torch.arange(0, n, 1 + n // 40)
    ref, want = lu.answers_ref(x[some], table, 1.0, torch.zeros(len(some), dtype=torch.int64), 9)
    assert torch.equal(ids.cpu()[some], want)
    for t, v in (("lse", lse), ("entropy", entropy), ("top_logp", logs)):
        du.within(v.cpu()[some], *ref[t], what=t)


@pytest.mark.parametrize("n", [30, 600])
def test_one_row_of_large_values_does_not_bring_all_of_the_table_up_again(ctx, n):
    """A call takes no more than a few times as long (all logits again in 64 bits: forty times and more)."""
    V, D, k = 300_000, 128, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x, table = (torch.randn(m, D, device="cuda", generator=g).bfloat16() for m in (n, V))
    times = []
    for outlier in (False, True):
        if outlier:
            table[V // 2, 7] = 10_000.0
        best = math.inf
        for _ in range(6):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            answers(ctx, x, table, 1.0, k)
            end.record()
            end.synchronize()
            best = min(best, start.elapsed_time(end))
        times.append(best)
    assert times[1] < 4 * times[0], times


def test_rows_in_turns(recd, ctx):
    """9000 rows of 1 000 003 go in two turns: every row is the same, and as a small call has it."""
    n, V, D = 9000, 1_000_003, 8
    x, table = torch.zeros(n, D, dtype=torch.bfloat16, device="cuda"), torch.randn(V, D, device="cuda").bfloat16()
    x[:, 0] = 1.0
    lse, entropy, ids, logs = answers(ctx, x, table, 1.0, 1)
    few = answers(ctx, x[:5], table, 1.0, 1)
    for a, b in ((lse, few[0]), (entropy, few[1]), (logs[:, 0], few[3][:, 0])):
        assert ((a.double() - b[0].double()).abs() <= 2 * SUM * (1 + b[0].double().abs())).all()
    assert (ids == few[2][0]).all()
