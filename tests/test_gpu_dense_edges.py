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
