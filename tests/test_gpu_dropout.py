"""Dropout from a counter, and its gradient, against 64 bits."""
import pytest
import torch

from tests import dense_util as du
from tests import layers_util as lu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def recd():
    from paper_2211_05239_amd import recd as mod
    return mod


@pytest.fixture(scope="module")
def ctx(recd):
    c = recd.Context(0)
    yield c
    c.close()


def check(recd, ctx, n, D, dt, p, seed, call, residual):
    x, g = du.rand((n, D), dt, 1, 1.5, 0.3), du.rand((n, D), dt, 2)
    r = du.rand((n, D), dt, 3) if residual else None
    drop = recd.Dropout(p, seed, call)
    out, gx = torch.full((n, D), float("nan"), dtype=x.dtype, device="cuda"), torch.full((n, D), float("nan"), dtype=x.dtype, device="cuda")
    ctx.dropout(x.cuda(), drop, out, residual=r.cuda() if residual else None)
    ctx.dropout_backward(g.cuda(), drop, gx)
    du.within(out, *lu.dropout_ref(x, p, seed, call, r), what="out")
    du.within(gx, *lu.dropout_ref(g, p, seed, call), what="grad_x")
    kept = lu.keep(n, D, p, seed, call)
    assert not gx.cpu()[~kept].any()
    return out, gx


# one row and piece, rows of half pieces (fp32), rows shorter and longer than a block, more pieces than the card's threads take at once
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("n,pieces", [(1, 1), (1, 3), (7, 2), (301, 5), (33, 129), (3, 4099), (2111, 64), (70_001, 9), (200_003, 1)])
def test_sizes(recd, ctx, dt, n, pieces, residual):
    check(recd, ctx, n, pieces * (4 if dt == "f32" else 8), dt, 0.1, 1234567, 3, residual)


@pytest.mark.parametrize("p", [0.0, 1e-6, 0.05, 0.5, 0.9, 65535 / 65536])
@pytest.mark.parametrize("seed,call", [(0, 0), (-1, -1), (1 << 63, 1 << 40), (0x0123456789ABCDEF, 0xFEDCBA9876543210)])
def test_probabilities_and_numbers(recd, ctx, p, seed, call):
    check(recd, ctx, 50, 72, "f32", p, seed, call, True)


def test_a_mask_is_one_of_rows_columns_and_calls(recd, ctx):
    """Not of the type, the number of rows, or the operator."""
    one = lambda dt, n, call: (lambda o: (ctx.dropout(torch.ones(n, 64, dtype=du.DT[dt], device="cuda"), recd.Dropout(0.3, 9, call), o), o != 0)[1])(  # noqa: E731
        torch.empty(n, 64, dtype=du.DT[dt], device="cuda"))
    a = one("f32", 500, 1)
    assert torch.equal(a, one("bf16", 500, 1)) and torch.equal(a[:77], one("f16", 77, 1)) and not torch.equal(a, one("f32", 500, 2))
    y = torch.empty(500, 64, device="cuda")
    ctx.dense(torch.zeros(500, 32, device="cuda"), torch.zeros(64, 32, device="cuda"), torch.ones(64, device="cuda"), y, dropout=recd.Dropout(0.3, 9, 1))
    assert torch.equal(a, y != 0)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_in_place(recd, ctx, dt):
    drop = recd.Dropout(0.2, 5, 6)
    x, r = du.rand((4099, 40), dt, 1).cuda(), du.rand((4099, 40), dt, 2).cuda()
    want, plain = torch.empty_like(x), torch.empty_like(x)
    ctx.dropout(x, drop, want, residual=r)
    ctx.dropout_backward(x, drop, plain)
    a, b, c = x.clone(), r.clone(), x.clone()
    ctx.dropout(a, drop, a, residual=r)
    ctx.dropout(x, drop, b, residual=b)
    ctx.dropout_backward(c, drop, c)
    assert du.same_bits(a, want) and du.same_bits(b, want) and du.same_bits(c, plain)


def test_what_is_dropped_is_zero_whatever_it_was(recd, ctx):
    drop = recd.Dropout(0.5, 5, 6)
    kept = lu.keep(100, 64, 0.5, 5, 6)
    for bad in (float("nan"), float("inf"), -float("inf")):
        x = torch.where(kept, 1.0, bad).cuda()
        out, gx = torch.empty_like(x), torch.empty_like(x)
        ctx.dropout(x, drop, out, residual=torch.ones_like(x))
        ctx.dropout_backward(x, drop, gx)
        assert torch.equal(out.cpu(), torch.where(kept, 3.0, 1.0)) and torch.equal(gx.cpu(), torch.where(kept, 2.0, 0.0))
    x = torch.where(kept, float("nan"), 1.0).cuda()
    ctx.dropout(x, drop, x)
    assert torch.equal(x.isnan().cpu(), kept)


def test_a_captured_step_takes_another_mask_at_each_replay(recd):
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c = recd.Context(0)
        step = torch.zeros(1, dtype=torch.int64, device="cuda")
        drop = recd.Dropout(0.4, 77, 100, step)
        x = du.rand((300, 64), "bf16", 1).cuda()
        out, gx = torch.empty_like(x), torch.empty_like(x)

        def work():
            c.dropout(x, drop, out)
            c.dropout_backward(x, drop, gx)
            step.add_(1)

        work()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            work()
        for i in range(1, 4):
            graph.replay()
            s.synchronize()
            assert int(step) == i + 1
            ref = lu.dropout_ref(x.cpu(), 0.4, 77, 100 + i)
            du.within(out, *ref)
            assert du.same_bits(out, gx)
            x.copy_(du.rand((300, 64), "bf16", i + 5))
        c.close()


def test_rows_beyond_32_bits_of_elements(recd, ctx):
    """2^32 elements and more: the last rows."""
    n, D = (1 << 32) // 4096 + 33, 4096
    x = torch.ones(n, D, dtype=torch.bfloat16, device="cuda")
    ctx.dropout(x, recd.Dropout(0.5, 3, 4), x)
    tail = x[-40:].cpu()
    assert torch.equal(tail != 0, lu.keep(40, D, 0.5, 3, 4, row0=n - 40))


def test_refusals(recd, ctx):
    import ctypes as C
    lib, h, bad = recd._lib, ctx._h, recd.RECD_EINVAL
    x = torch.zeros(4, 64, device="cuda")
    p, m = x.data_ptr(), C.byref(recd._Mask(0.1, 1, 2, None))
    assert lib.recd_dropout(h, 4, 64, 0, None, p, None, p) == bad
    for prob in (1.0, -0.5, float("nan"), 0.999999):
        assert lib.recd_dropout(h, 4, 64, 0, C.byref(recd._Mask(prob, 1, 2, None)), p, None, p) == bad
        assert lib.recd_dropout_backward(h, 4, 64, 0, C.byref(recd._Mask(prob, 1, 2, None)), p, p) == bad
    assert lib.recd_dropout(h, 4, 64, 0, C.byref(recd._Mask(0.1, 1, 2, p + 4)), p, None, p) == bad
    assert lib.recd_dropout(h, -1, 64, 0, m, p, None, p) == bad
    assert lib.recd_dropout(h, 1 << 48, 64, 0, m, p, None, p) == bad
    for D, dt in ((0, 0), (3, 0), (4, 1), (65540, 0), (64, 3)):
        assert lib.recd_dropout(h, 4, D, dt, m, p, None, p) == bad
    assert lib.recd_dropout(h, 4, 64, 0, m, None, None, p) == bad and lib.recd_dropout(h, 4, 64, 0, m, p, None, None) == bad
    assert lib.recd_dropout(h, 4, 64, 0, m, p + 4, None, p) == bad and lib.recd_dropout(h, 4, 64, 0, m, p, p + 8, p) == bad
    assert b"aligned" in lib.recd_last_error(h)
    assert lib.recd_dropout(h, 0, 64, 0, m, None, None, None) == recd.RECD_OK
    with pytest.raises(AssertionError):
        ctx.dropout(x, recd.Dropout(0.1, 1, 2, torch.zeros(1, device="cuda")), x)
