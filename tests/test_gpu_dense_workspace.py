"""What the dense operators' calls take of the workspace is what their sizing functions say, and a context created with it keeps its
workspace, so that graphs may go on using it."""
import pytest
import torch

from tests import dense_util as du

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def recd():
    from paper_2211_05239_amd import recd as mod
    return mod


def taken(recd, hint, use):
    """Bytes of device memory that a context holds once `use` has gone over it."""
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    c = recd.Context(0, workspace_hint_bytes=hint)
    use(c)
    torch.cuda.synchronize()
    after = torch.cuda.mem_get_info()[0]
    c.close()
    return before - after


def check(recd, want, use):
    assert want > 1 << 20   # (small ones do not show beside what every context holds)
    use(recd_ctx := recd.Context(0))
    recd_ctx.close()        # (kernels are loaded)
    held = taken(recd, want, use)
    assert held == taken(recd, want, lambda c: None)     # enough
    assert held == taken(recd, 0, use)                   # and no more than is needed


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,V,D", [(64, 600_000, 128), (300, 300_000, 64), (2000, 90_000, 64), (300_000, 1000, 32)])
def test_vocab_loss(recd, dt, n, V, D):
    dtype = du.DT[dt]
    x, table = torch.zeros(n, D, dtype=dtype, device="cuda"), torch.zeros(V, D, dtype=dtype, device="cuda")
    t, gl = torch.zeros(n, dtype=torch.int64, device="cuda"), torch.zeros(n, device="cuda")
    loss, lse, mean = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, D, device="cuda")
    gx, gt = torch.empty_like(x), torch.empty_like(table)

    def use(c):
        c.vocab_loss(x, table, t, 1.0, loss, lse)
        c.vocab_loss(x, table, t, 1.0, loss, lse, mean)
        c.vocab_loss_backward(x, table, t, 1.0, lse, mean, gl, gx, gt)

    check(recd, recd.vocab_loss_workspace_bytes(n, V, D, dtype), use)


# (single rows whose keys are split; short lists, listed; long ones)
@pytest.mark.parametrize("lq,lk,H,G,d", [([1] * 64, [9000] * 64, 8, 2, 128), ([3, 0, 9] * 90_000, [3, 0, 9] * 90_000, 4, 4, 8),
                                         ([4000] * 40 + [1], [4000] * 40 + [1], 16, 8, 64)])
def test_list_attention(recd, lq, lk, H, G, d):
    qo, ko = (torch.tensor([0] + lens).cumsum(0).cuda() for lens in (lq, lk))
    Q, K = sum(lq), sum(lk)
    q, g = torch.zeros(Q, H, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(Q, H, d, dtype=torch.bfloat16, device="cuda")
    k, v = torch.zeros(K, G, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(K, G, d, dtype=torch.bfloat16, device="cuda")
    out, lse, gq, gk, gv = torch.empty_like(q), torch.empty(Q, H, device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)

    def use(c):
        c.list_attention(q, k, v, qo, ko, max(lq), max(lk), out, lse, scale=1.0)
        c.list_attention_backward(q, k, v, qo, ko, max(lq), max(lk), out, lse, g, gq, gk, gv, scale=1.0)

    check(recd, recd.list_attention_workspace_bytes(H, G, d, q.dtype, len(lq), max(lq), max(lk), Q, K), use)


def test_layer_norm(recd):
    n, D = 100_000, 1024
    x, w = torch.zeros(n, D, device="cuda"), torch.zeros(D, device="cuda")
    stats, y = torch.empty(n, 2, device="cuda"), torch.empty_like(x)
    gw, gb = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")

    def use(c):
        c.layer_norm(x, w, w, 1e-5, y, stats)
        c.layer_norm_backward(x, w, stats, x, y, gw, gb)

    check(recd, recd.layer_norm_workspace_bytes(n, D, x.dtype), use)


def test_a_graph_beside_larger_calls(recd):
    """A small step is captured on a context with room for a large one, whose call comes between the replays."""
    D, V, n, many = 64, 3000, 200, 50_000
    x, table = du.rand((many, D), "bf16", 1).cuda(), du.rand((V, D), "bf16", 2).cuda()
    t, gl = (torch.arange(many) % V).cuda(), torch.ones(many, device="cuda")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        room = max(recd.vocab_loss_workspace_bytes(m, V, D, x.dtype) for m in (n, many))
        c = recd.Context(0, workspace_hint_bytes=room)

        def outputs(m):
            return torch.zeros(m, device="cuda"), torch.zeros(m, device="cuda"), torch.zeros(m, D, device="cuda"), torch.zeros_like(x[:m]), torch.zeros_like(table)

        def step(m, o):
            c.vocab_loss(x[:m], table, t[:m], 1.0, o[0], o[1], o[2])
            c.vocab_loss_backward(x[:m], table, t[:m], 1.0, o[1], o[2], gl[:m], o[3], o[4])

        small, want, large = outputs(n), outputs(n), outputs(many)
        step(n, want)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step(n, small)
        for _ in range(3):
            step(many, large)
            for o in small:
                o.fill_(float("nan"))
            graph.replay()
            s.synchronize()
            for a, b in zip(small, want):
                assert torch.equal(a, b)
        c.close()


def test_refusals(recd):
    import ctypes as C
    out, lib = C.c_size_t(7), recd._lib
    assert lib.recd_vocab_loss_workspace_bytes(0, 4, 8, 64, 0, None) == recd.RECD_EINVAL
    assert lib.recd_vocab_loss_workspace_bytes(-1, 4, 8, 64, 0, C.byref(out)) == recd.RECD_EINVAL
    assert lib.recd_vocab_loss_workspace_bytes(99, 4, 8, 64, 0, C.byref(out)) == recd.RECD_EHIP
    assert lib.recd_vocab_loss_workspace_bytes(0, -4, 8, 64, 0, C.byref(out)) == recd.RECD_EINVAL
    assert lib.recd_layer_norm_workspace_bytes(0, 4, 3, 0, C.byref(out)) == recd.RECD_EINVAL
    assert lib.recd_list_attention_workspace_bytes(0, None, C.byref(out)) == recd.RECD_EINVAL
    with pytest.raises(recd.RecdError):
        recd.list_attention_workspace_bytes(3, 2, 64, torch.float32, 1, 4, 4, 4, 4)
    assert out.value == 7
    assert recd.vocab_loss_workspace_bytes(0, 0, 64, torch.float32) == 0
    assert recd.list_attention_workspace_bytes(2, 2, 64, torch.float32, 0, 0, 0, 0, 0) <= 4096
