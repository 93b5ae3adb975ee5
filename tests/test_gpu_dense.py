"""Dense layers and their gradients against 64 bits, and what the calls refuse."""
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


def data(n, K, N, dt, seed=1, bias=True, residual=False):
    x, w, g = du.rand((n, K), dt, seed), du.rand((N, K), dt, seed + 1, K ** -0.5), du.rand((n, N), dt, seed + 2)
    return x, w, du.rand((N,), "f32", seed + 3, 0.3) if bias else None, du.rand((n, N), dt, seed + 4) if residual else None, g


def strided(t, wide, fill=0.0):
    """t on the device, in the middle of wider rows (whose other elements hold `fill`)."""
    if t is None or not wide:
        return t.cuda() if t is not None else None
    big = torch.full((t.shape[0], t.shape[1] + 48), fill, dtype=t.dtype, device="cuda")
    big[:, 16:-32] = t.cuda()
    return big[:, 16:-32]


def run(recd, ctx, x, w, b, r, g, act="none", p=0.0, wide=False, kept=False, stream_inputs=None):
    n, N, nan = x.shape[0], w.shape[0], float("nan")
    xd, rd, gd, wd = strided(x, wide, nan), strided(r, wide, nan), strided(g, wide, nan), w.cuda()
    bd = b.cuda() if b is not None else None
    y, gx = strided(torch.full_like(g, nan), wide, 5.0), strided(torch.full_like(x, nan), wide, 5.0)
    gw, gb = torch.full_like(wd, nan), torch.full((N,), nan, device="cuda")
    sums = torch.full((n, N), nan, device="cuda") if kept else None
    drop = recd.Dropout(p, 99, 7) if p else None
    ctx.dense(xd, wd, bd, y, act=act, dropout=drop, residual=rd, sums=sums)
    ctx.dense_backward(xd, wd, bd, gd, gx, gw, gb, act=act, dropout=drop, sums=sums)
    torch.cuda.synchronize()
    if wide:
        for t in (y, gx):  # what lies between the rows stays
            if t.shape[0] > 1:
                between = t.as_strided((t.shape[0] - 1, 48), (t.stride(0), 1), t.storage_offset() + t.shape[1])
                assert (between == 5.0).all()
    out = {"y": y, "grad_x": gx, "grad_w": gw, "grad_bias": gb}
    return {**out, "sums": sums} if kept else out


def check(recd, ctx, x, w, b, r, g, act="none", p=0.0, **how):
    got = run(recd, ctx, x, w, b, r, g, act, p, **how)
    ref = lu.dense_ref(x, w, b, act, p, 99, 7, r, g)
    for k, v in got.items():
        du.within(v, *ref[k], what=k)
    return got


# rows: few (one, a tile's edges, the last of the form for few), then tiles; widths: one piece, a tile's edges, ends inside a tile
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 33, 64, 65, 127, 300])
@pytest.mark.parametrize("K,N", [(8, 8), (24, 136), (64, 64), (200, 72), (520, 40)])
def test_sizes(recd, ctx, dt, n, K, N):
    check(recd, ctx, *data(n, K, N, dt), "gelu", 0.1)


# one to eight rows in blocks of four and eight features: ends of the contraction, of the features, of the rows, rows too long for it
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [1, 3, 4, 5, 8, 9])
@pytest.mark.parametrize("K,N", [(2048, 8), (2056, 24), (4096, 200), (4104, 4104), (8192, 72), (8200, 16), (20_000, 40)])
def test_few_rows_of_long_ones(recd, ctx, dt, n, K, N):
    check(recd, ctx, *data(n, K, N, dt, residual=True), "silu", 0.1, kept=True)


def test_few_rows_of_widths_of_four(recd, ctx):
    for n in (1, 4, 7):
        for K, N in ((2052, 4), (4100, 12), (2044, 60)):
            check(recd, ctx, *data(n, K, N, "f32", residual=True), "gelu", 0.1, wide=True)


# sums of many splits: of the rows for w's gradient, of the features for x's
@pytest.mark.parametrize("dt,n,K,N", [("bf16", 20_011, 64, 24), ("f16", 5003, 8, 8), ("f32", 9001, 20, 12), ("f32", 2999, 132, 68),
                                      ("bf16", 70, 24, 16_384), ("f32", 65, 4, 8188)])
def test_many_splits(recd, ctx, dt, n, K, N):
    check(recd, ctx, *data(n, K, N, dt), "none", 0.1)


# ... and of a long contraction, in the layer itself and where z is made again
@pytest.mark.parametrize("act,p", [("gelu", 0.1), ("none", 0.0)])
@pytest.mark.parametrize("dt,n,K,N", [("f32", 27, 5844, 60), ("bf16", 65, 8192, 40), ("f16", 100, 3080, 8), ("f32", 70, 2052, 4)])
def test_many_splits_of_a_long_contraction(recd, ctx, dt, n, K, N, act, p):
    check(recd, ctx, *data(n, K, N, dt, residual=True), act, p)
    check(recd, ctx, *data(n, K, N, dt, bias=False), act, p, wide=True, kept=True)


# fp32 tiles of few columns, in each product: tiles of 64 would take the card once more
@pytest.mark.parametrize("n,K,N", [(18_307, 68, 140), (18_307, 140, 68), (70, 140, 18_308)])
def test_narrow_tiles(recd, ctx, n, K, N):
    check(recd, ctx, *data(n, K, N, "f32", residual=True), "silu", 0.1)


@pytest.mark.parametrize("n,K,N", [(1, 4, 4), (37, 12, 20), (100, 36, 4), (129, 68, 132), (1000, 4, 100)])
def test_widths_of_four(recd, ctx, n, K, N):
    """fp32 rows that end in half a piece of eight."""
    check(recd, ctx, *data(n, K, N, "f32", residual=True), "silu", 0.3)


# tiles of 256 and 128 (many of them), a long contraction in splits, with a tail, and a gradient of w of many tiles
@pytest.mark.parametrize("dt,n,K,N", [("bf16", 8197, 72, 2056), ("f16", 5000, 264, 1032), ("bf16", 100, 4104, 72), ("f32", 70, 4100, 36),
                                      ("f32", 2100, 100, 2052), ("bf16", 77, 4096, 4104), ("f32", 90, 2052, 2052), ("bf16", 30_001, 16, 24),
                                      ("f32", 20_003, 24, 16)])
def test_cuts(recd, ctx, dt, n, K, N):
    x, w, b, r, g = data(n, K, N, dt)
    a = check(recd, ctx, x, w, b, r, g, "silu", 0.0)
    again = run(recd, ctx, x, w, b, r, g, "silu", 0.0)
    for k in a:
        assert du.same_bits(a[k], again[k]), k


# few rows and a long contraction: split, with tails, or by tiles
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [1, 7, 16, 17, 50])
@pytest.mark.parametrize("K,N", [(4104, 72), (8200, 16), (2048, 520), (1032, 24)])
def test_few_rows_of_many_elements(recd, ctx, dt, n, K, N):
    x, w, b, r, g = data(n, K, N, dt, residual=True)
    a = check(recd, ctx, x, w, b, r, g, "gelu", 0.1, kept=True)
    again = run(recd, ctx, x, w, b, r, g, "gelu", 0.1, kept=True)
    for k in a:
        assert du.same_bits(a[k], again[k]), k


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("n", [40, 200])
@pytest.mark.parametrize("p,residual,bias", [(0.0, False, False), (0.0, True, True), (0.5, True, False), (0.1, False, True)])
def test_epilogues(recd, ctx, dt, act, n, p, residual, bias):
    x, w, b, r, g = data(n, 96, 104, dt, bias=bias, residual=residual)
    check(recd, ctx, x, w, b, r, g, act, p)
    check(recd, ctx, x, w, b, r, g, act, p, wide=True, kept=True)


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("size", [3.0, 30.0])
def test_far_from_zero(recd, ctx, act, size):
    """Sums of any size: tails of the activations, on both sides."""
    x, w, b, r, g = data(300, 64, 64, "f32")
    check(recd, ctx, x * size, w, b, r, g, act)
    z = torch.linspace(-120, 120, 4096)[None]
    w0, y = torch.zeros(4096, 4), torch.empty(1, 4096, device="cuda")
    ctx.dense(torch.zeros(1, 4, device="cuda"), w0.cuda(), z[0].cuda(), y, act=act)
    ref, _, bound, _, _ = lu._act(act, z.double())
    du.within(y, ref, bound)


def test_any_of_the_gradients(recd, ctx):
    x, w, b, r, g = (t.cuda() if t is not None else None for t in data(300, 64, 72, "bf16"))
    for how in (dict(), dict(act="gelu"), dict(act="gelu", dropout=recd.Dropout(0.2, 1, 2)), dict(dropout=recd.Dropout(0.2, 1, 2))):
        full = [torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)]
        ctx.dense_backward(x, w, b, g, *full, **how)
        for mask in range(1, 8):
            some = [torch.full_like(t, 3.0) if mask >> i & 1 else None for i, t in enumerate(full)]
            ctx.dense_backward(x, w, b, g, *some, **how)
            for a, want in zip(some, full):
                assert a is None or du.same_bits(a, want)
        ctx.dense_backward(x, w, b, g, **how)


def test_without_rows(recd, ctx):
    w, b = torch.ones(24, 16, device="cuda"), torch.ones(24, device="cuda")
    x, y = torch.empty(0, 16, device="cuda"), torch.empty(0, 24, device="cuda")
    gw, gb = torch.full_like(w, 7.0), torch.full_like(b, 7.0)
    for act in ("none", "gelu"):
        ctx.dense(x, w, b, y, act=act)
        ctx.dense_backward(x, w, b, y, x.clone(), gw.fill_(7.0), gb.fill_(7.0), act=act)
        assert not gw.any() and not gb.any()


@pytest.mark.parametrize("n", [20, 200])
def test_the_residual_may_be_the_result(recd, ctx, n):
    x, w, b, r, g = (t.cuda() for t in data(n, 64, 72, "f16", residual=True))
    want, there = torch.empty_like(r), r.clone()
    ctx.dense(x, w, b, want, residual=r, act="gelu")
    ctx.dense(x, w, b, there, residual=there, act="gelu")
    assert du.same_bits(there, want)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [33, 300])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_rows_that_are_not_finite_stay_by_themselves(recd, ctx, dt, n, bad):
    """In a row's last element too, in widths that end inside a tile; not in the sums over rows, of course."""
    x, w, b, r, g = data(n, 72, 40, dt)
    want = run(recd, ctx, x, w, b, r, g, "gelu")
    x, g = x.clone(), g.clone()
    x[3, 71], x[n - 1, 0], g[5, 39] = bad, bad, bad
    got = run(recd, ctx, x, w, b, r, g, "gelu")
    rows = torch.ones(n, dtype=torch.bool, device="cuda")
    rows[3] = rows[n - 1] = False
    assert du.same_bits(got["y"][rows], want["y"][rows])
    rows[5] = False
    assert du.same_bits(got["grad_x"][rows], want["grad_x"][rows])
    if bad != bad:
        assert got["y"][3].isnan().all() and got["grad_x"][5].isnan().all()


def test_a_weight_that_is_not_finite_stays_with_its_feature(recd, ctx):
    for n in (20, 200):
        x, w, b, r, g = data(n, 72, 40, "bf16")
        w[39, 71] = float("inf")
        y = torch.empty(n, 40, dtype=torch.bfloat16, device="cuda")
        ctx.dense(x.cuda(), w.cuda(), b.cuda(), y)
        assert y[:, :39].isfinite().all() and not y[:, 39].isfinite().any()


@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
def test_gradients_against_differences(recd, ctx, act):
    """Central differences of sum(g * y) in fp32: off by the differences' own rounding (2^-24 of the sum's terms over h) and by h^2."""
    x, w, b, r, g = data(6, 8, 8, "f32")
    drop = recd.Dropout(0.25, 3, 1)
    grads = [torch.empty_like(t).cuda() for t in (x, w, b)]
    ctx.dense_backward(x.cuda(), w.cuda(), b.cuda(), g.cuda(), *grads, act=act, dropout=drop)
    h = 2.0 ** -7

    def value():
        y = torch.empty(6, 8, device="cuda")
        ctx.dense(x.cuda(), w.cuda(), b.cuda(), y, act=act, dropout=drop)
        return float((y.double().cpu() * g.double()).sum())

    for t, got in zip((x, w, b), grads):
        flat = t.view(-1)
        for i in range(flat.numel()):
            old = float(flat[i])
            flat[i] = old + h
            up = value()
            flat[i] = old - h
            down = value()
            flat[i] = old
            assert abs((up - down) / (2 * h) - float(got.view(-1)[i])) < 5e-3, (act, i)


def test_another_stream_and_two_contexts(recd, ctx):
    x, w, b, r, g = data(999, 64, 136, "bf16")
    want = run(recd, ctx, x, w, b, r, g, "gelu", 0.1)
    streams = [torch.cuda.Stream() for _ in range(2)]
    got, contexts = [], []
    for s in streams:
        with torch.cuda.stream(s):
            contexts.append(recd.Context(0))
            got.append(run(recd, contexts[-1], x, w, b, r, g, "gelu", 0.1))
    torch.cuda.synchronize()
    for one in got:
        for k in want:
            assert du.same_bits(one[k], want[k]), k
    for c in contexts:
        c.close()


def test_a_graph_beside_larger_calls(recd):
    """A small step is captured on a context with room for a large one, whose calls come between the replays."""
    n, many, K, N = 200, 9000, 64, 264
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step = torch.zeros(1, dtype=torch.int64, device="cuda")
        drop = recd.Dropout(0.1, 5, 6, step)
        x, w, b, r, g = (t.cuda() for t in data(many, K, N, "bf16", residual=True))
        room = max(recd.dense_workspace_bytes(m, K, N, x.dtype, "gelu", drop) for m in (n, many))
        c = recd.Context(0, workspace_hint_bytes=room)

        def outputs(m):
            return [torch.zeros(m, N, dtype=x.dtype, device="cuda"), torch.zeros(m, K, dtype=x.dtype, device="cuda"), torch.zeros_like(w), torch.zeros_like(b)]

        def work(m, o):
            c.dense(x[:m], w, b, o[0], act="gelu", dropout=drop, residual=r[:m])
            c.dense_backward(x[:m], w, b, g[:m], *o[1:], act="gelu", dropout=drop)

        small, want, large = outputs(n), outputs(n), outputs(many)
        work(n, small)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            work(n, small)
        for i in range(3):
            step.fill_(i)
            work(many, large)
            work(n, want)
            for o in small:
                o.fill_(float("nan"))
            graph.replay()
            s.synchronize()
            for a, e in zip(small, want):
                assert du.same_bits(a, e)
        c.close()


@pytest.mark.parametrize("dt,n,K,N,act,p", [("bf16", 3000, 4096, 136, "gelu", 0.1), ("f32", 100, 2048, 2048, "silu", 0.0),
                                            ("f16", 50_000, 128, 128, "none", 0.0), ("bf16", 50, 4096, 1024, "none", 0.2)])
def test_workspace(recd, dt, n, K, N, act, p):
    """What a pair of calls takes is what the sizing function says."""
    dtype = du.DT[dt]
    x, w, b = torch.zeros(n, K, dtype=dtype, device="cuda"), torch.zeros(N, K, dtype=dtype, device="cuda"), torch.zeros(N, device="cuda")
    y, g, sums = (torch.zeros(n, N, dtype=t, device="cuda") for t in (dtype, dtype, torch.float32))
    gx, gw, gb = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    drop = recd.Dropout(p, 1, 2) if p else None

    def use(c):
        c.dense(x, w, b, y, act=act, dropout=drop, sums=sums)
        c.dense_backward(x, w, b, g, gx, gw, gb, act=act, dropout=drop)
        c.dense_backward(x, w, b, g, gx, gw, gb, act=act, dropout=drop, sums=sums)
        c.dense_backward(x, w, b, g, None, gw, None, act=act, dropout=drop, sums=sums)

    want = recd.dense_workspace_bytes(n, K, N, dtype, act, drop)

    def taken(hint, use):
        torch.cuda.synchronize()
        before = torch.cuda.mem_get_info()[0]
        c = recd.Context(0, workspace_hint_bytes=hint)
        use(c)
        torch.cuda.synchronize()
        after = torch.cuda.mem_get_info()[0]
        c.close()
        return before - after

    taken(0, use)  # (kernels are loaded)
    held = taken(want, use)
    assert held == taken(want, lambda c: None)
    assert abs(held - taken(0, use)) <= 1 << 21  # (memory is handed out in pieces of this size)


def test_rows_far_apart(recd, ctx):
    """Rows nearly 16 MiB apart: offsets beyond 32 bits."""
    n, K, N, stride = 300, 64, 40, (1 << 23) - 8
    x, w, b, r, g = data(n, K, N, "bf16")
    far = torch.zeros((n - 1) * stride + 64, dtype=torch.bfloat16, device="cuda")
    want = run(recd, ctx, x, w, b, r, g, "gelu")
    gx = torch.empty(n, K, dtype=torch.bfloat16, device="cuda")
    gw, gb, y = torch.empty(N, K, dtype=torch.bfloat16, device="cuda"), torch.empty(N, device="cuda"), torch.empty(n, N, dtype=torch.bfloat16, device="cuda")
    xs = far.as_strided((n, K), (stride, 1))
    xs.copy_(x)
    for m in (40, n):
        ctx.dense(xs[:m], w.cuda(), b.cuda(), y[:m], act="gelu")
        assert du.same_bits(y[:20], want["y"][:20]) or m < n
    assert du.same_bits(y, want["y"])
    ctx.dense_backward(xs, w.cuda(), b.cuda(), g.cuda(), gx, gw, gb, act="gelu")
    for a, k in ((gx, "grad_x"), (gw, "grad_w"), (gb, "grad_bias")):
        assert du.same_bits(a, want[k]), k
    ctx.dense_backward(x.cuda(), w.cuda(), b.cuda(), g.cuda(), xs, None, None, act="gelu")
    assert du.same_bits(xs, want["grad_x"])
    ys = far.as_strided((n, N), (stride, 1))
    ctx.dense(x.cuda(), w.cuda(), b.cuda(), ys, act="gelu")
    assert du.same_bits(ys, want["y"])
    ys.copy_(g)
    ctx.dense_backward(x.cuda(), w.cuda(), b.cuda(), ys, gx, gw, gb, act="none")
    plain = run(recd, ctx, x, w, b, r, g, "none")
    for a, k in ((gx, "grad_x"), (gw, "grad_w"), (gb, "grad_bias")):
        assert du.same_bits(a, plain[k]), k


def test_more_rows_than_one_launch_takes(recd, ctx):
    """2^30 rows and more go in turns; the mask counts on over them."""
    n, K = (1 << 30) + 300, 8
    x = torch.full((n, K), 1.0, dtype=torch.bfloat16, device="cuda")
    w = torch.eye(K, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros(n, K, dtype=torch.bfloat16, device="cuda")
    x[-1] = 3.0
    ctx.dense(x, w, None, y, dropout=recd.Dropout(0.5, 3, 4))
    assert torch.equal((y[-400:] != 0).cpu(), lu.keep(400, K, 0.5, 3, 4, row0=n - 400))
    assert set(y[-1].tolist()) <= {0.0, 6.0} and set(y[-2].tolist()) <= {0.0, 2.0}
    assert torch.equal((y[:400] != 0).cpu(), lu.keep(400, K, 0.5, 3, 4))


def test_refusals(recd, ctx):
    import ctypes as C
    lib, h, bad = recd._lib, ctx._h, recd.RECD_EINVAL
    t = torch.zeros(64 * 64, device="cuda")
    p = t.data_ptr()

    def layer(n=4, K=64, N=64, dt=0, act=0, xs=64, rs=64, ys=64, mask=None):
        return C.byref(recd._Dense(n, K, N, dt, act, xs, rs, ys, mask))

    def forward(a, x=p, w=p, b=None, r=None, s=None, y=p):
        return lib.recd_dense(h, a, x, w, b, r, s, y)

    assert lib.recd_dense(h, None, p, p, None, None, None, p) == bad
    for a in (layer(n=-1), layer(K=3), layer(N=0), layer(dt=3), layer(act=9), layer(xs=63), layer(xs=60), layer(ys=32), layer(xs=66),
              layer(xs=1 << 22), layer(ys=1 << 22), layer(mask=C.pointer(recd._Mask(1.0, 0, 0, None)))):
        assert forward(a) == bad
    assert forward(layer(rs=32), r=p) == bad
    assert forward(layer(), x=None) == bad and forward(layer(), w=None) == bad and forward(layer(), y=None) == bad
    assert forward(layer(), x=p + 4) == bad and forward(layer(), r=p + 8) == bad and forward(layer(), s=p + 4) == bad
    assert forward(layer(), b=p + 2) == bad
    assert b"aligned" in lib.recd_last_error(h)
    assert forward(layer(n=0), x=None, w=None, y=None) == recd.RECD_OK

    def backward(a, x=p, w=p, s=None, g=p, gs=64, gx=p, gxs=64, gw=p, gb=None):
        return lib.recd_dense_backward(h, a, x, w, None, s, g, gs, gx, gxs, gw, gb)

    assert backward(layer(), g=None) == bad and backward(layer(), x=None) == bad and backward(layer(), w=None) == bad
    assert backward(layer(), gs=60) == bad and backward(layer(), gxs=60) == bad and backward(layer(), gw=p + 4) == bad
    assert backward(layer(), s=p + 4) == bad and backward(layer(), gb=p + 1) == bad and backward(layer(xs=2)) == bad
    x = torch.zeros(4, 64, device="cuda")
    with pytest.raises(AssertionError):
        ctx.dense(x, torch.zeros(64, 32, device="cuda"), None, torch.zeros(4, 64, device="cuda"))
    with pytest.raises(AssertionError):
        ctx.dense(x.t(), torch.zeros(64, 4, device="cuda"), None, torch.zeros(64, 64, device="cuda"))
    with pytest.raises(KeyError):
        ctx.dense(x, torch.zeros(64, 64, device="cuda"), None, torch.zeros(4, 64, device="cuda"), act="tanh")
