"""Dense layers where a mask, a type's range or the rows' distance could lose something: dropped places that are not finite, fp16 gradients
far below and above what fp16 holds, few rows far apart."""
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


# z in one launch, by splits with the rows' kernel behind it, and by many splits
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("n,K,N", [(70, 64, 72), (65, 4104, 72), (27, 5844, 60)])
@pytest.mark.parametrize("kept", [False, True])
def test_dropped_places_that_are_not_finite(recd, ctx, dt, act, n, K, N, kept):
    """z is infinite or NaN in features all of whose rows are dropped: nothing of it reaches a result."""
    if dt != "f32" and N % 8:
        K, N = K // 8 * 8, 64
    p, seed, call = 0.97, 5, 9
    drop = recd.Dropout(p, seed, call)
    x, w, r, g = (t.cuda() for t in (du.rand((n, K), dt, 1), du.rand((N, K), dt, 2, K ** -0.5), du.rand((n, N), dt, 4), du.rand((n, N), dt, 3)))
    b = du.rand((N,), "f32", 6).cuda()
    gone = (~lu.keep(n, N, p, seed, call)).all(0).nonzero()[:, 0]
    assert len(gone) >= 3

    def run(b):
        y, sums = torch.empty_like(g), torch.empty(n, N, device="cuda") if kept else None
        grads = [torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)]
        ctx.dense(x, w, b, y, act=act, dropout=drop, residual=r, sums=sums)
        ctx.dense_backward(x, w, b, g, *grads, act=act, dropout=drop, sums=sums)
        return [y] + grads

    want = run(b)
    for v in want:
        assert v.isfinite().all()
    bad = b.clone()
    bad[gone] = torch.tensor([float("inf"), -float("inf"), float("nan")], device="cuda").repeat(len(gone))[:len(gone)]
    for a, e in zip(run(bad), want):
        assert du.same_bits(a, e)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "gelu", "silu"])
def test_dropped_gradients_that_are_not_finite(recd, ctx, dt, act):
    n, K, N = 70, 64, 72
    drop = recd.Dropout(0.5, 8, 3)
    gone = ~lu.keep(n, N, 0.5, 8, 3).cuda()
    x, w, g = (t.cuda() for t in (du.rand((n, K), dt, 1), du.rand((N, K), dt, 2, 0.1), du.rand((n, N), dt, 3)))
    out = []
    for bad in (0.0, float("inf"), float("nan")):
        grads = [torch.empty_like(x), torch.empty_like(w), torch.empty(N, device="cuda")]
        ctx.dense_backward(x, w, None, torch.where(gone, bad, g), *grads, act=act, dropout=drop)
        out.append(grads)
    for other in out[1:]:
        for a, e in zip(other, out[0]):
            assert du.same_bits(a, e)


def grads_ref(x, w, b, act, p, seed, call, g):
    """lu.dense_ref's gradients of a layer of fp16, with other bounds: gz is rounded to fp16 times a power of two that brings the largest
    |g| / (1 - p) * 1.13 (1.13: the steepest slope) to between 2^14 and 2^15.  Below 2^-14 steps are of 2^-24, so a rounding is at most
    2^-25 there: 2^-39 of that largest value."""
    ref = lu.dense_ref(x, w, b, act, p, seed, call, None, g)
    n, N = g.shape
    by = 65536.0 / (65536 - lu.cut(p))
    into = 2.0 ** -39 * 1.13 * by * float(g.double()[g.isfinite()].abs().max()) - 2.0 ** -25  # in the place of dense_ref's absolute term
    xa, wa = x.double().abs(), w.double().abs()
    gx, gw = ref["grad_x"], ref["grad_w"]
    return {"grad_x": (gx[0], gx[1] + into * wa.sum(0)[None]), "grad_w": (gw[0], gw[1] + into * xa.sum(0)[None]), "grad_bias": ref["grad_bias"]}


# one launch for both gradients; w's by splits, added up by eight waves; x's by splits; tiles of 256 (two launches)
@pytest.mark.parametrize("n,K,N", [(70, 64, 72), (5003, 8, 8), (70, 24, 16_384), (8197, 264, 1032), (300, 520, 40)])
@pytest.mark.parametrize("act,p", [("gelu", 0.1), ("silu", 0.0), ("none", 0.5), ("relu", 0.3)])
@pytest.mark.parametrize("size", ["small", "large"])
def test_fp16_gradients_beyond_its_range(recd, ctx, n, K, N, act, p, size):
    """Gradients of a few of fp16's smallest steps, or beyond its largest value once they are divided by 1 - p: x and w bring the results
    back into range, one of them at a time."""
    drop = recd.Dropout(p, 3, 4) if p else None
    g = du.rand((n, N), "f16", 1, 2.0 ** -22) if size == "small" else du.rand((n, N), "f16", 1).clamp(-2, 2) * 30_000
    up = 2.0 ** 8 if size == "small" else 2.0 ** -12
    for name in ("grad_x", "grad_w"):
        # z's size is 1 in both: (x, w) = (1 / up, up) for grad_x = gz w, (up, 1 / up) for grad_w = gz^T x
        by_w = up if name == "grad_x" else 1 / up
        x, w = du.rand((n, K), "f16", 2, 1 / by_w), du.rand((N, K), "f16", 3, by_w * K ** -0.5)
        b = du.rand((N,), "f32", 4, 0.3)
        ref = grads_ref(x, w, b, act, p, 3, 4, g)
        got = {"grad_x": torch.empty_like(x).cuda(), "grad_w": torch.empty_like(w).cuda(), "grad_bias": torch.empty(N, device="cuda")}
        for kept in (False, True):
            sums = None
            if kept:
                sums = torch.empty(n, N, device="cuda")
                ctx.dense(x.cuda(), w.cuda(), b.cuda(), torch.empty(n, N, dtype=x.dtype, device="cuda"), act=act, dropout=drop, sums=sums)
            ctx.dense_backward(x.cuda(), w.cuda(), b.cuda(), g.cuda(), *got.values(), act=act, dropout=drop, sums=sums)
            assert got[name].isfinite().all() and float(got[name].abs().max()) > 2.0 ** -16
            for k in (name, "grad_bias"):
                du.within(got[k], *ref[k], what=(k, kept))


def test_fp16_gradients_in_a_graph(recd):
    """The gradients' size is that of the replay, not of the capture; zeros and infinities do not set it."""
    n, K, N = 200, 64, 264
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        drop = recd.Dropout(0.1, 5, 6)
        x, w, g0 = (t.cuda() for t in (du.rand((n, K), "f16", 1, 0.01), du.rand((N, K), "f16", 2, 10.0), du.rand((n, N), "f16", 3)))
        c = recd.Context(0, workspace_hint_bytes=recd.dense_workspace_bytes(n, K, N, x.dtype, "gelu", drop))
        g = g0.clone()
        small, want = ([torch.zeros_like(x), torch.zeros_like(w), torch.zeros(N, device="cuda")] for _ in range(2))

        def work(o):
            c.dense_backward(x, w, None, g, *o, act="gelu", dropout=drop)

        work(small)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            work(small)
        infinite = g0 * 2.0 ** -20
        infinite[3, 5] = float("inf")
        for t in (g0 * 2.0 ** -20, torch.zeros_like(g0), g0 * 2.0 ** 10, infinite, g0):
            g.copy_(t)
            work(want)
            for o in small:
                o.fill_(float("nan"))
            graph.replay()
            s.synchronize()
            for a, e in zip(small, want):
                assert torch.equal(a[a.isfinite()], e[e.isfinite()]) and torch.equal(a.isfinite(), e.isfinite())
            if not t.any():
                assert not any(o.any() for o in small)
        g.copy_(infinite)
        work(small)
        g[3, 5] = 0
        work(want)
        rows = torch.arange(n, device="cuda") != 3
        assert du.same_bits(small[0][rows], want[0][rows])
        c.close()


@pytest.mark.parametrize("m", [1, 5, 16, 40, 64])
def test_few_rows_far_apart(recd, ctx, m):
    """Rows nearly 16 MiB apart in the forms of few rows: the bits of rows that lie densely."""
    K, N, stride = 64, 40, (1 << 23) - 8
    x, w, b, r = (t.cuda() for t in (du.rand((m, K), "bf16", 1), du.rand((N, K), "bf16", 2, 0.1), du.rand((N,), "f32", 3), du.rand((m, N), "bf16", 4)))
    want, y = torch.empty_like(r), torch.full_like(r, float("nan"))
    ctx.dense(x, w, b, want, act="gelu", residual=r)
    far = torch.zeros((m - 1) * stride + 64, dtype=torch.bfloat16, device="cuda")
    xs = far.as_strided((m, K), (stride, 1))
    xs.copy_(x)
    ctx.dense(xs, w, b, y, act="gelu", residual=r)
    assert du.same_bits(y, want)
    ys = far.as_strided((m, N), (stride, 1))
    ys.copy_(r)
    ctx.dense(x, w, b, ys, act="gelu", residual=ys)
    assert du.same_bits(ys, want)


def test_distances_whose_bytes_pass_64_bits(recd, ctx):
    import ctypes as C
    t = torch.zeros(64 * 64, device="cuda")
    p = t.data_ptr()
    for far in (1 << 62, (1 << 62) + 64, (1 << 63) - 64):
        for place in range(3):
            strides = [64, 64, 64]
            strides[place] = far
            a = recd._Dense(4, 64, 64, 0, 0, *strides, None)
            assert recd._lib.recd_dense(ctx._h, C.byref(a), p, p, None, p, None, p) == recd.RECD_EINVAL
        a = recd._Dense(4, 64, 64, 0, 0, 64, 64, 64, None)
        assert recd._lib.recd_dense_backward(ctx._h, C.byref(a), p, p, None, None, p, far, p, 64, p, None) == recd.RECD_EINVAL
        assert recd._lib.recd_dense_backward(ctx._h, C.byref(a), p, p, None, None, p, 64, p, far, p, None) == recd.RECD_EINVAL


@pytest.mark.parametrize("n,K,N", [(300, 64, 72), (5003, 8, 8), (70, 24, 16_384)])
@pytest.mark.parametrize("wide", [False, True])
def test_any_of_the_fp16_gradients(recd, ctx, n, K, N, wide):
    """Each by itself has the bits that it has beside the others, also from rows inside of wider ones that hold infinities."""
    x, w, b, g = (t.cuda() for t in (du.rand((n, K), "f16", 1, 0.01), du.rand((N, K), "f16", 2, 10.0), du.rand((N,), "f32", 3), du.rand((n, N), "f16", 4, 2.0 ** -18)))
    if wide:
        big = torch.full((n, N + 48), float("inf"), dtype=g.dtype, device="cuda")
        big[:, 16:-32] = g
        g = big[:, 16:-32]
    for how in (dict(act="gelu"), dict(act="silu", dropout=recd.Dropout(0.2, 1, 2)), dict(dropout=recd.Dropout(0.2, 1, 2)), dict()):
        full = [torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)]
        ctx.dense_backward(x, w, b, g, *full, **how)
        assert all(t.isfinite().all() and t.any() for t in full)
        for mask in range(1, 8):
            some = [torch.full_like(t, 3.0) if mask >> i & 1 else None for i, t in enumerate(full)]
            ctx.dense_backward(x, w, b, g, *some, **how)
            for a, want in zip(some, full):
                assert a is None or du.same_bits(a, want)
