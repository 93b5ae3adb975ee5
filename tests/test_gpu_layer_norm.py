"""Layer norm and its gradients against 64 bits, and what the calls refuse."""
import pytest
import torch

from tests import dense_util as du

pytestmark = pytest.mark.gpu
EPS = 1e-5


def run(ctx, x, w, b, g, eps=EPS):
    dev = lambda t: None if t is None else t.cuda()  # noqa: E731
    x, w, b, g = dev(x), dev(w), dev(b), dev(g)
    n, D = x.shape
    nan = float("nan")
    got = {"y": torch.full_like(x, nan), "grad_x": torch.full_like(x, nan), "grad_weight": torch.full((D,), nan, device="cuda"),
           "grad_bias": torch.full((D,), nan, device="cuda")}
    stats = torch.full((n, 2), nan, device="cuda")
    ctx.layer_norm(x, w, b, eps, got["y"], stats)
    plain = torch.full_like(x, nan)
    ctx.layer_norm(x, w, b, eps, plain)
    ctx.layer_norm_backward(x, w, stats, g, got["grad_x"], got["grad_weight"], got["grad_bias"])
    torch.cuda.synchronize()
    assert du.same_bits(plain, got["y"])
    return got


@pytest.fixture(scope="module")
def ctx():
    from paper_2211_05239_amd import recd
    c = recd.Context(0)
    yield c
    c.close()


# rows of 1 to 256 pieces: one lane, idle lanes, one to four pieces a lane
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("pieces", [1, 2, 3, 5, 8, 24, 64, 65, 100, 129, 192, 193, 256])
def test_rows_of_every_width(ctx, dt, pieces):
    D = pieces * (4 if dt == "f32" else 8)
    n = 77
    x, g = du.rand((n, D), dt, pieces, 1.5, 0.3), du.rand((n, D), dt, pieces + 1)
    w, b = du.rand((D,), "f32", 3, 0.3, 1.0), du.rand((D,), "f32", 4, 0.3)
    ref = du.norm_ref(x, w, b, EPS, g)
    for k, v in run(ctx, x, w, b, g).items():
        du.within(v, *ref[k], what=k)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 31, 4097, 70_001])
def test_numbers_of_rows(ctx, dt, n):
    D = 40
    x, g = du.rand((n, D), dt, n, 2.0, -1.0), du.rand((n, D), dt, n + 1)
    w, b = du.rand((D,), "f32", 3), du.rand((D,), "f32", 4)
    ref = du.norm_ref(x, w, b, EPS, g)
    got = run(ctx, x, w, b, g)
    for k, v in got.items():
        du.within(v, *ref[k], what=k)
    again = run(ctx, x, w, b, g)
    for k in got:
        assert torch.equal(got[k], again[k]), k


def test_without_weight_and_bias_and_rows(ctx):
    x, g = du.rand((50, 64), "f32", 1), du.rand((50, 64), "f32", 2)
    ref = du.norm_ref(x, None, None, EPS, g)
    got = run(ctx, x, None, None, g)
    for k, v in got.items():
        du.within(v, *ref[k], what=k)
    # sums over no rows are zero
    x0, stats = torch.empty(0, 64, device="cuda"), torch.empty(0, 2, device="cuda")
    gw, gb = torch.full((64,), 7.0, device="cuda"), torch.full((64,), 7.0, device="cuda")
    ctx.layer_norm(x0, None, None, EPS, x0.clone(), stats)
    ctx.layer_norm_backward(x0, None, stats, x0.clone(), x0.clone(), gw, gb)
    assert not gw.any() and not gb.any()


def test_sums_are_optional_and_rows_may_be_replaced(ctx):
    x, g = du.rand((300, 96), "bf16", 1).cuda(), du.rand((300, 96), "bf16", 2).cuda()
    w, b = du.rand((96,), "f32", 3).cuda(), du.rand((96,), "f32", 4).cuda()
    got = run(ctx, x.cpu(), w.cpu(), b.cpu(), g.cpu())
    stats, y = torch.empty(300, 2, device="cuda"), x.clone()
    ctx.layer_norm(y, w, b, EPS, y, stats)
    assert torch.equal(y, got["y"])
    gw = torch.empty(96, device="cuda")
    there = g.clone()
    ctx.layer_norm_backward(x, w, stats, there, there, gw)
    assert torch.equal(there, got["grad_x"]) and torch.equal(gw, got["grad_weight"])
    there = g.clone()
    ctx.layer_norm_backward(x, w, stats, there, there)
    assert torch.equal(there, got["grad_x"])


def test_constant_rows_and_large_means(ctx):
    """The variance is taken about the mean: a mean a thousand times the spread costs its rounding, not its square."""
    x = torch.cat([du.rand((40, 128), "f32", 1, 1.0, 1000.0), torch.full((3, 128), 5.0)])
    w, b, g = du.rand((128,), "f32", 3), du.rand((128,), "f32", 4), du.rand((43, 128), "f32", 5)
    ref = du.norm_ref(x, w, b, EPS, g)
    got = run(ctx, x, w, b, g)
    for k in ("y", "grad_x"):
        du.within(got[k][:40], ref[k][0][:40], ref[k][1][:40], what=k)
    assert torch.equal(got["y"][40:].cpu(), b.expand(3, 128))


def test_a_row_that_is_not_finite_stays_by_itself(ctx):
    x = du.rand((64, 32), "f32", 1)
    x[5, 3], x[9, 0] = float("nan"), float("inf")
    w, b, g = du.rand((32,), "f32", 3), du.rand((32,), "f32", 4), du.rand((64, 32), "f32", 5)
    got = run(ctx, x, w, b, g)
    rows = torch.ones(64, dtype=torch.bool)
    rows[5] = rows[9] = False
    assert got["y"][5].isnan().all() and got["y"][9].isnan().any()
    assert got["y"][rows.cuda()].isfinite().all() and got["grad_x"][rows.cuda()].isfinite().all()


@pytest.mark.parametrize("dt", ["f32"])
def test_gradients_against_differences(ctx, dt):
    """Central differences of sum(g * y) in fp32: off by the differences' own rounding (about 2^-24 * |sum| / h) and h^2."""
    x, g = du.rand((4, 8), dt, 1), du.rand((4, 8), dt, 2)
    w, b = du.rand((8,), "f32", 3, 0.3, 1.0), du.rand((8,), "f32", 4)
    got = run(ctx, x, w, b, g)
    h = 2.0 ** -7

    def value(x, w, b):
        y = torch.empty_like(x).cuda()
        ctx.layer_norm(x.cuda(), w.cuda(), b.cuda(), EPS, y)
        return float((y.double().cpu() * g.double()).sum())

    for name, t in (("grad_x", x), ("grad_weight", w), ("grad_bias", b)):
        flat = t.view(-1)
        for i in range(flat.numel()):
            old = float(flat[i])
            flat[i] = old + h
            up = value(x, w, b)
            flat[i] = old - h
            down = value(x, w, b)
            flat[i] = old
            assert abs((up - down) / (2 * h) - float(got[name].view(-1)[i])) < 5e-3, (name, i)


def test_another_stream(ctx):
    from paper_2211_05239_amd import recd
    s = torch.cuda.Stream()
    x, g = du.rand((999, 64), "bf16", 1), du.rand((999, 64), "bf16", 2)
    w, b = du.rand((64,), "f32", 3), du.rand((64,), "f32", 4)
    want = run(ctx, x, w, b, g)
    with torch.cuda.stream(s):
        c = recd.Context(0)
        got = run(c, x, w, b, g)
        s.synchronize()
        c.close()
    for k in want:
        assert torch.equal(got[k], want[k]), k


def test_refusals(ctx):
    from paper_2211_05239_amd import recd
    lib, h = recd._lib, ctx._h
    x = torch.zeros(4, 64, device="cuda")
    p, st = x.data_ptr(), torch.zeros(8, device="cuda").data_ptr()
    bad = recd.RECD_EINVAL
    assert lib.recd_layer_norm(None, 4, 64, 0, p, None, None, EPS, p, None) == bad
    assert lib.recd_layer_norm(h, -1, 64, 0, p, None, None, EPS, p, None) == bad
    for D, dt in ((0, 0), (3, 0), (1028, 0), (4, 1), (2056, 2), (64, 3)):
        assert lib.recd_layer_norm(h, 4, D, dt, p, None, None, EPS, p, None) == bad
        assert lib.recd_layer_norm_backward(h, 4, D, dt, p, None, st, p, p, None, None) == bad
    assert lib.recd_layer_norm(h, 4, 64, 0, None, None, None, EPS, p, None) == bad
    assert lib.recd_layer_norm(h, 4, 64, 0, p + 4, None, None, EPS, p, None) == bad
    assert b"aligned" in lib.recd_last_error(h)
    assert lib.recd_layer_norm_backward(h, 4, 64, 0, p, None, None, p, p, None, None) == bad
    assert lib.recd_layer_norm_backward(h, 4, 64, 0, p, None, st, p, p + 8, None, None) == bad
    assert lib.recd_layer_norm(h, 0, 64, 0, None, None, None, EPS, None, None) == recd.RECD_OK


@pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16, torch.float64])
def test_statistics_of_another_type_are_refused(ctx, dt):
    """They are eight bytes a row, whatever the rows' type."""
    x = du.rand((40, 32), "bf16", 1).cuda()
    with pytest.raises(AssertionError):
        ctx.layer_norm(x, None, None, 1e-5, torch.empty_like(x), torch.zeros(40, 2, dtype=dt, device="cuda"))
    ctx.layer_norm(x, None, None, 1e-5, torch.empty_like(x), torch.zeros(40, 2, device="cuda"))


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,D", [(1, 16), (37, 8), (5000, 128), (9001, 520)])   # (the last: several rows a wave, three pieces a lane)
def test_in_place(ctx, dt, n, D):
    """y may be x, and grad_x may be grad_y: the same bits, row after row of a lane's."""
    x, g = du.rand((n, D), dt, 1), du.rand((n, D), dt, 2)
    w, b = du.rand((D,), "f32", 3), du.rand((D,), "f32", 4)
    want = run(ctx, x, w, b, g)
    y, stats, x = x.cuda(), torch.empty(n, 2, device="cuda"), x.cuda()
    ctx.layer_norm(y, w.cuda(), b.cuda(), EPS, y, stats)
    gx = g.cuda()
    gw, gb = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    ctx.layer_norm_backward(x, w.cuda(), stats, gx, gx, gw, gb)
    for got, k in ((y, "y"), (gx, "grad_x"), (gw, "grad_weight"), (gb, "grad_bias")):
        assert du.same_bits(got, want[k]), k
