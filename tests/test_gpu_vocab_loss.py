"""Softmax cross entropy against a table, its gradients, and what the calls refuse, against 64 bits."""
import pytest
import torch

from tests import dense_util as du

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2211_05239_amd import recd
    c = recd.Context(0)
    yield c
    c.close()


def data(n, V, D, dt, seed, std=1.5, ignored=True):
    x, table = du.rand((n, D), dt, seed), du.rand((V, D), dt, seed + 1, std / D ** 0.5)
    g = torch.Generator().manual_seed(seed + 2)
    t = torch.randint(0, V, (n,), generator=g)
    if ignored:
        t[::5] = -1
    t[1::7] = V - 1
    return x, table, t, du.rand((n,), "f32", seed + 3, 0.5, 1.0)


def run(ctx, x, table, t, scale, gl, device=True):
    x, table, t, gl = (a.cuda() for a in (x, table, t, gl)) if device else (x, table, t, gl)
    n, D = x.shape
    nan = float("nan")
    got = {"loss": torch.full((n,), nan, device="cuda"), "lse": torch.full((n,), nan, device="cuda"),
           "grad_x": torch.full_like(x, nan), "grad_table": torch.full_like(table, nan)}
    mean = torch.full((n, D), nan, device="cuda")
    ctx.vocab_loss(x, table, t, scale, got["loss"], got["lse"], mean)
    loss, lse = torch.full((n,), nan, device="cuda"), torch.full((n,), nan, device="cuda")
    ctx.vocab_loss(x, table, t, scale, loss, lse)
    ctx.vocab_loss_backward(x, table, t, scale, got["lse"], mean, gl, got["grad_x"], got["grad_table"])
    torch.cuda.synchronize()
    return got, {"loss": loss, "lse": lse}


def check(ctx, x, table, t, scale, gl):
    ref = du.loss_ref(x, table, t, scale, gl)
    got, without = run(ctx, x, table, t, scale, gl)
    for k, v in got.items():
        du.within(v, *ref[k], what=k)
    for k, v in without.items():
        du.within(v, *ref[k], what=k + " without the gradient")
    return got


# rows: one, a tile's edges, few (waves share them) and many; vocabularies: one row, a tile's edges, several splits
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,V,D", [(1, 1, 16), (1, 31, 64), (33, 32, 24), (5, 33, 128), (64, 129, 40), (65, 1000, 96),
                                   (128, 257, 128), (129, 999, 72), (300, 4097, 64), (257, 130, 200), (40, 3001, 256),
                                   (700, 640, 256)])
def test_sizes(ctx, dt, n, V, D):
    check(ctx, *data(n, V, D, dt, n + V)[:3], 1.0, data(n, V, D, dt, n + V)[3])


# small tables and many rows: the table's gradient is cut across its rows, and their parts are added up
@pytest.mark.parametrize("dt,n,V,D", [("f32", 2000, 9000, 64), ("f16", 3000, 9001, 128), ("bf16", 2999, 5000, 96)])
def test_table_rows_that_several_blocks_share(ctx, dt, n, V, D):
    x, table, t, gl = data(n, V, D, dt, 21)
    a = check(ctx, x, table, t, 1.0, gl)
    b, _ = run(ctx, x, table, t, 1.0, gl)
    for k in a:
        assert torch.equal(a[k], b[k]), k


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [-0.7, 0.05, 20.0])
def test_scales(ctx, dt, scale):
    """A negative scale turns the maximum round; a large one makes single probabilities near 1."""
    x, table, t, gl = data(150, 500, 64, dt, 9)
    check(ctx, x, table, t, scale, gl)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_many_rows_share_a_target(ctx, dt):
    """One table row is almost every row's target: what is left of the sum beside the targets' weights has to be right."""
    x, table, t, gl = data(600, 300, 64, dt, 3, ignored=False)
    t[:550] = 17
    check(ctx, x, table, t, 1.0, gl)


@pytest.mark.parametrize("power", [-30, 10])
def test_fp16_weights_of_any_size(ctx, power):
    """Small and large weights of the loss neither vanish nor overflow inside; the result's own range decides."""
    x, table, t, gl = data(90, 400, 64, "f16", 4)
    gl = gl * 2.0 ** power
    ref = du.loss_ref(x, table, t, 1.0, gl)
    got, _ = run(ctx, x, table, t, 1.0, gl)
    for k in ("grad_x", "grad_table"):
        du.within(got[k], *ref[k], what=k)


def test_rows_without_any_target(ctx):
    x, table, t, gl = data(70, 200, 64, "bf16", 5)
    t[:] = -100
    got = check(ctx, x, table, t, 1.0, gl)
    assert not got["loss"].any() and not got["grad_x"].any() and not got["grad_table"].any()


def test_a_target_beyond_the_table(ctx):
    from paper_2211_05239_amd import recd
    x, table, t, gl = data(20, 50, 32, "f32", 6)
    t[3] = 50
    got = check(ctx, x, table, t, 1.0, gl)
    assert got["loss"][3] == 0 and not got["grad_x"][3].any()
    ctx.set_option(recd.RECD_OPT_VALIDATE, 1)
    try:
        with pytest.raises(recd.RecdError, match="target") as e:
            run(ctx, x, table, t, 1.0, gl)
        assert e.value.status == recd.RECD_EBOUNDS
        t[3] = 49
        run(ctx, x, table, t, 1.0, gl)
    finally:
        ctx.set_option(recd.RECD_OPT_VALIDATE, 0)


def test_large_logits_do_not_overflow(ctx):
    """Logits of several thousands, rising along the vocabulary, so that the running maximum moves again and again."""
    x, table, _, gl = data(130, 700, 64, "f32", 8)
    x, table = x.abs() * 20, table.abs() * torch.linspace(0, 40, 700)[:, None]
    t = torch.arange(130) * 5 % 700
    check(ctx, x.contiguous(), table.contiguous(), t, 1.0, gl)


def test_a_row_that_is_not_finite_stays_by_itself(ctx):
    x, table, t, gl = data(200, 300, 64, "f32", 8)
    x[7, 2] = float("nan")
    t[7] = -1
    got, _ = run(ctx, x, table, t, 1.0, gl)
    others = torch.arange(200, device="cuda") != 7
    assert got["lse"][7].isnan() and got["lse"][others].isfinite().all() and got["grad_x"][others].isfinite().all()


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,V,D", [(90, 300, 64), (700, 3000, 128), (300, 500, 200)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_rows_without_a_target_may_hold_anything(ctx, dt, n, V, D, bad):
    """Neither their elements nor their losses' weights reach a gradient."""
    x, table, t, gl = data(n, V, D, dt, 8)
    ref = du.loss_ref(x, table, t, 1.0, gl)
    x[t < 0, ::2] = bad
    gl[t < 0] = bad
    got, _ = run(ctx, x, table, t, 1.0, gl)
    du.within(got["grad_table"], *ref["grad_table"], what="grad_table")
    du.within(got["grad_x"], *ref["grad_x"], what="grad_x")
    has = t >= 0
    du.within(got["loss"].cpu(), *ref["loss"], what="loss")
    du.within(got["lse"].cpu()[has], ref["lse"][0][has], ref["lse"][1][has], what="lse")


def test_same_bits_again(ctx):
    x, table, t, gl = data(500, 5000, 128, "bf16", 11)
    a, _ = run(ctx, x, table, t, 1.0, gl)
    b, _ = run(ctx, x, table, t, 1.0, gl)
    for k in a:
        assert torch.equal(a[k], b[k]), k


def test_only_one_gradient(ctx):
    x, table, t, gl = (a.cuda() for a in data(140, 900, 64, "f16", 12))
    want, _ = run(ctx, x, table, t, 1.0, gl, device=False)
    mean = torch.empty(140, 64, device="cuda")
    loss, lse = torch.empty(140, device="cuda"), torch.empty(140, device="cuda")
    ctx.vocab_loss(x, table, t, 1.0, loss, lse, mean)
    gx, gt = torch.empty_like(x), torch.empty_like(table)
    ctx.vocab_loss_backward(x, table, t, 1.0, lse, mean, gl, gx, None)
    ctx.vocab_loss_backward(x, table, t, 1.0, lse, None, gl, None, gt)
    assert torch.equal(gx, want["grad_x"]) and torch.equal(gt, want["grad_table"])


def test_no_rows(ctx):
    table = du.rand((40, 64), "bf16", 1).cuda()
    x, e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(0, device="cuda")
    t = torch.empty(0, dtype=torch.int64, device="cuda")
    gt = torch.full_like(table, 3.0)
    ctx.vocab_loss(x, table, t, 1.0, e, e)
    ctx.vocab_loss_backward(x, table, t, 1.0, e, torch.empty(0, 64, device="cuda"), e, x.clone(), gt)
    assert not gt.any()


def test_gradients_against_differences(ctx):
    """Central differences of the weighted loss in fp32: off by the losses' rounding over the step and its square."""
    x, table, t, gl = data(5, 9, 8, "f32", 13, ignored=False)
    got, _ = run(ctx, x, table, t, 1.0, gl)
    h = 2.0 ** -7

    def value():
        loss, lse = torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
        ctx.vocab_loss(x.cuda(), table.cuda(), t.cuda(), 1.0, loss, lse)
        return float((loss.double().cpu() * gl.double()).sum())

    for name, a in (("grad_x", x), ("grad_table", table)):
        flat = a.view(-1)
        for i in range(flat.numel()):
            old = float(flat[i])
            flat[i] = old + h
            up = value()
            flat[i] = old - h
            down = value()
            flat[i] = old
            assert abs((up - down) / (2 * h) - float(got[name].view(-1)[i])) < 2e-3, (name, i)


def test_a_table_beyond_2_to_31_elements(ctx):
    """Rows whose positions pass 32 bits: the last rows hold the only logits that count."""
    V, D = 17_000_000, 128
    table = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda")
    x = du.rand((6, D), "bf16", 1, 1.0)
    tail = du.rand((1000, D), "bf16", 2, 1.0)
    table[V - 1000:] = tail.cuda()
    t = torch.tensor([V - 1, V - 1000, 3, V - 5, V - 500, -1])
    got, _ = run(ctx, x.cuda(), table, t.cuda(), 2.0, torch.ones(6).cuda(), device=False)
    z = 2.0 * (x.double() @ tail.double().t())
    lse = torch.logsumexp(torch.cat([z, torch.full((6, 1), float(torch.tensor(V - 1000.0).log()), dtype=torch.float64)], 1), 1)
    picked = torch.tensor([z[0, 999], z[1, 0], 0.0, z[3, 995], z[4, 500], 0.0], dtype=torch.float64)
    assert (got["lse"].double().cpu() - lse).abs().max() < 1e-4
    assert (got["loss"].double().cpu() - torch.where(t >= 0, lse - picked, 0.0)).abs().max() < 1e-4
    p = (z - lse[:, None]).exp()
    g = torch.tensor([1, 1, 1, 1, 1, 0], dtype=torch.float64)
    w = p * g[:, None]
    for i, at in enumerate((999, 0, None, 995, 500)):
        if at is not None:
            w[i, at] -= 1.0
    ref = 2.0 * (w.t() @ x.double())
    assert (got["grad_table"][V - 1000:].double().cpu() - ref).norm() < 6e-3 * ref.norm()
    ref3 = -2.0 * x[2].double()
    assert (got["grad_table"][3].double().cpu() - ref3).norm() < 6e-3 * ref3.norm()


def test_replayed_from_a_graph(ctx):
    """A captured step on a context that has seen the sizes, replayed with other work and synchronisations in between."""
    from paper_2211_05239_amd import recd
    x, table, t, gl = (a.cuda() for a in data(300, 2000, 64, "f16", 14))
    n, D = x.shape
    want, _ = run(ctx, x, table, t, 1.0, gl, device=False)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c = recd.Context(0)
        out = [torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, D, device="cuda"),
               torch.zeros_like(x), torch.zeros_like(table)]

        def step():
            c.vocab_loss(x, table, t, 1.0, out[0], out[1], out[2])
            c.vocab_loss_backward(x, table, t, 1.0, out[1], out[2], gl, out[3], out[4])

        step()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
        for i in range(4):
            for o in out:
                o.fill_(float("nan"))
            graph.replay()
            s.synchronize()
            for o, k in ((out[0], "loss"), (out[1], "lse"), (out[3], "grad_x"), (out[4], "grad_table")):
                assert torch.equal(o, want[k]), (i, k)
            run(c, x, table, t, 1.0, gl, device=False)
        c.close()


def test_refusals(ctx):
    from paper_2211_05239_amd import recd
    lib, h = recd._lib, ctx._h
    a = torch.zeros(4096, device="cuda")
    p = a.data_ptr()

    def forward(n=4, V=8, D=64, dt=0, x=p, table=p, t=p, scale=1.0, loss=p, lse=p, ctx_=h):
        return lib.recd_vocab_loss(ctx_, n, V, D, dt, x, table, t, scale, loss, lse, None)

    def backward(n=4, V=8, D=64, dt=0, lse=p, mean=p, gl=p, gx=p, gt=p, scale=1.0):
        return lib.recd_vocab_loss_backward(h, n, V, D, dt, p, p, p, scale, lse, mean, gl, gx, gt)

    for kw in (dict(ctx_=None), dict(n=-1), dict(V=-1), dict(V=0), dict(V=1 << 31), dict(n=1 << 31), dict(D=0), dict(D=6),
               dict(D=260), dict(D=12, dt=1), dict(dt=3), dict(x=None), dict(table=None), dict(t=None), dict(loss=None),
               dict(lse=None), dict(x=p + 4), dict(table=p + 8), dict(scale=0.0), dict(scale=float("nan")),
               dict(scale=float("inf"))):
        assert forward(**kw) == recd.RECD_EINVAL, kw
    for kw in (dict(D=260), dict(lse=None), dict(gl=None), dict(mean=None), dict(gx=None, gt=None), dict(gx=p + 4),
               dict(gt=p + 2), dict(V=0), dict(scale=0.0)):
        assert backward(**kw) == recd.RECD_EINVAL, kw
    assert forward(n=0, x=None, t=None, loss=None, lse=None) == recd.RECD_OK


def confident(dt, seed, n=400, D=64):
    """Rows that their model predicts well, 1 - p_t from a tenth to 1e-4: every target a table row of its own, behind one that
    points the same way and stands 4 to 13 powers of two below it."""
    half = 500
    table = du.rand((2 * half, D), dt, seed)
    table[:half] = (table[half:].double() * 0.7).to(table.dtype)
    t = torch.randperm(half, generator=torch.Generator().manual_seed(seed))[:n] + half
    w = table[t].double()
    z = torch.linspace(10.0, 30.0, n, dtype=torch.float64)[:, None]
    x = (w * z / w.square().sum(1, keepdim=True)).to(table.dtype)
    return x, table, t, du.rand((n,), "f32", seed + 3, 0.1, 1.0)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("n,scale", [(400, 1.0), (200, 1.0), (400, -1.0)])   # (many rows, few rows, a negative scale)
def test_rows_that_are_predicted_well(ctx, dt, n, scale):
    """Gradients of a row in proportion to what is left to learn, 1 - p_t, not to 1.

    The target's weight in the table's gradient is g (p_t - 1), subtracted before anything is rounded, and the row's gradient the
    others' probabilities, each with its own rounding u; what fp32 leaves of a logit, dz, counts in full beside 1 - p_t.  A logit
    is a sum of D / 16 matrix products of exact terms, each off by 2 E of what it has summed, and the steps of its exponent."""
    x, table, t, gl = confident(dt, 31, n)
    x = x if scale > 0 else -x
    got = check(ctx, x, table, t, scale, gl)
    u = du.U[x.dtype]
    xd, w = x.double(), table.double()
    z = scale * (xd @ w.t())
    lse = torch.logsumexp(z, 1)
    p = (z - lse[:, None]).exp()
    rows = torch.arange(n)
    pt = p[rows, t]
    left = p.clone()
    left[rows, t] = 0.0
    rest = left.sum(1)                                                # 1 - p_t
    assert rest.min() < 2e-4 and 0.04 < rest.max() < 0.2
    D = x.shape[1]
    dz = 2 * du.E * (D / 16 + 4) * (xd.abs() * w[t].abs()).sum(1) + 8 * du.E * (z[rows, t].abs() + lse.abs())
    g = gl.double()
    weights = left * g[:, None]
    weights[rows, t] = -g * rest
    want = scale * (weights.t() @ xd)[t]
    off = (got["grad_table"].double().cpu()[t] - want).norm(dim=1)
    shares = ((left * g[:, None]).t() @ xd.abs())[t].norm(dim=1) + (g * rest)[:, None].mul(xd.abs()).norm(dim=1)
    bound = u * want.norm(dim=1) + u * shares + g * pt * dz * xd.norm(dim=1)
    assert (off <= bound).all(), float((off / bound).max())
    want = scale * g[:, None] * (left @ w - rest[:, None] * w[t])
    off = (got["grad_x"].double().cpu() - want).norm(dim=1)
    bound = u * want.norm(dim=1) + g * ((u * (left @ w.abs() + rest[:, None] * w[t].abs())).norm(dim=1) + (dz + 8 * du.E) * w[t].norm(dim=1))
    assert (off <= bound).all(), float((off / bound).max())


def infinite_elements(ctx, dt, n, V, D, where):
    """A table row that holds infinities at `where`, against rows that are positive there: its logits are -inf."""
    x, table, t, gl = data(n, V, D, dt, 8)
    x[:, where] = x[:, where].abs() + 0.1
    t[t == 11] = 12
    table[11, where] = -float("inf")
    fine = table.clone()
    fine[11, where] = -1000.0 if dt != "f32" else -1e6
    ref = du.loss_ref(x, fine, t, 1.0, gl)
    x, table, t, gl = (a.cuda() for a in (x, table, t, gl))
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ctx.vocab_loss(x, table, t, 1.0, loss, lse)
    du.within(loss, *ref["loss"], what="loss")
    du.within(lse, *ref["lse"], what="lse")
    gt = torch.empty_like(table)
    ctx.vocab_loss_backward(x, table, t, 1.0, lse, None, gl, None, gt)
    du.within(gt, *ref["grad_table"], what="grad_table")


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,V,D", [(60, 400, 64), (300, 700, 128)])
def test_infinite_elements_of_a_table_row(ctx, dt, n, V, D):
    """Rows without a target leave such a row's gradient alone, too."""
    infinite_elements(ctx, dt, n, V, D, slice(5, 8))


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_a_row_with_a_target_that_is_not_finite(ctx, dt):
    """What is wrong with a row that counts shows in its loss, its gradient and the table's."""
    x, table, t, gl = data(200, 300, 64, dt, 8)
    x[8, 2] = float("nan")
    t[8] = 3
    got, _ = run(ctx, x, table, t, 1.0, gl)
    assert got["loss"][8].isnan() and got["grad_x"][8].isnan().all() and got["grad_table"].isnan().all()
    others = torch.arange(200, device="cuda") != 8
    assert got["loss"][others].isfinite().all() and got["grad_x"][others].isfinite().all()


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,V,D", [(60, 400, 40), (300, 700, 72), (300, 500, 200)])
def test_infinite_last_elements_of_a_table_row(ctx, dt, n, V, D):
    """However much wider than the row a tile is."""
    infinite_elements(ctx, dt, n, V, D, slice(-3, None))


def test_more_rows_than_a_launch_holds(ctx):
    """2^26 rows and a few: 2^32 threads, at 64 a row, are more than one launch takes."""
    n, V, D = (1 << 26) + 5, 33, 8
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    x = torch.empty(n, D, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    t = torch.randint(-3, V, (n,), device="cuda", generator=gen)
    table = du.rand((V, D), "bf16", 2).cuda()
    gl = torch.full((n,), 1.0, device="cuda")
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    mean = torch.empty(n, D, device="cuda")
    gx, gt = torch.full_like(x, float("nan")), torch.full_like(table, float("nan"))
    ctx.vocab_loss(x, table, t, 1.0, loss, lse, mean)
    ctx.vocab_loss_backward(x, table, t, 1.0, lse, mean, gl, gx, gt)
    del mean
    for a in (0, (1 << 24) - 500, (1 << 25) - 500, 3 * (1 << 24) - 500, n - 1000):
        rows = slice(a, a + 1000)
        ref = du.loss_ref(x[rows].cpu(), table.cpu(), t[rows].cpu(), 1.0, gl[rows].cpu())
        for got, k in ((loss, "loss"), (lse, "lse"), (gx, "grad_x")):
            du.within(got[rows], *ref[k], what=f"{k} from {a}")
    want, size = torch.zeros(V, D, dtype=torch.float64, device="cuda"), torch.zeros(V, D, dtype=torch.float64, device="cuda")
    for a in range(0, n, 1 << 22):
        xs, ts = x[a:a + (1 << 22)].double(), t[a:a + (1 << 22)]
        w = torch.softmax(xs @ table.double().t(), 1)
        w[torch.arange(len(ts), device="cuda"), ts.clamp(min=0)] -= 1.0
        w[ts < 0] = 0.0
        want += w.t().contiguous() @ xs
        size += w.abs().t().contiguous() @ xs.abs()
    # weights rounded by u, and sums of n terms in order, whose roundings are of random sign: off by 4 E sqrt(n) of the terms' sizes
    assert ((gt.double() - want).abs() <= (du.U[gt.dtype] + 4 * du.E * n ** 0.5) * size).all()


def test_more_table_rows_than_a_launch_holds_are_refused(ctx):
    from paper_2211_05239_amd import recd
    lib, h = recd._lib, ctx._h
    a = torch.zeros(4096, device="cuda")
    p = a.data_ptr()
    assert lib.recd_vocab_loss(h, 4, (1 << 31) - 511, 64, 0, p, p, p, 1.0, p, p, None) == recd.RECD_EINVAL


def test_gradient_of_an_absent_table_is_refused(ctx):
    """Also without rows of x, where the table's gradient is zeros."""
    from paper_2211_05239_amd import recd
    lib, h = recd._lib, ctx._h
    a = torch.zeros(4096, device="cuda")
    p = a.data_ptr()
    assert lib.recd_vocab_loss_backward(h, 0, 8, 64, 0, None, None, None, 1.0, None, None, None, None, p) == recd.RECD_EINVAL
    assert lib.recd_vocab_loss_backward(h, 0, 8, 64, 0, None, p, None, 1.0, None, None, None, None, p) == recd.RECD_OK
