"""Attention inside lists, its gradients, and what the calls refuse, against 64 bits."""
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


def offsets(lens):
    return torch.cat([torch.zeros(1, dtype=torch.int64), torch.tensor(lens, dtype=torch.int64).cumsum(0)])


def run(ctx, q, k, v, qo, ko, how, g=None, max_q=None, max_k=None):
    dev = lambda t: t.cuda() if isinstance(t, torch.Tensor) else t  # noqa: E731
    q, k, v, g, qo, ko = (dev(t) for t in (q, k, v, g, qo, ko))
    how = {n: dev(x) for n, x in how.items()}
    max_q = int(qo.diff().max()) if max_q is None else max_q
    max_k = int(ko.diff().max()) if max_k is None else max_k
    nan = float("nan")
    got = {"out": torch.full(q.shape, nan, dtype=q.dtype, device="cuda"), "lse": torch.full(q.shape[:2], nan, device="cuda")}
    ctx.list_attention(q, k, v, qo, ko, max_q, max_k, got["out"], got["lse"], **how)
    plain = torch.full(q.shape, nan, dtype=q.dtype, device="cuda")
    ctx.list_attention(q, k, v, qo, ko, max_q, max_k, plain, **how)
    assert du.same_bits(plain, got["out"])
    if g is not None:
        for n, t in (("grad_q", q), ("grad_k", k), ("grad_v", v)):
            got[n] = torch.full(t.shape, nan, dtype=q.dtype, device="cuda")
        ctx.list_attention_backward(q, k, v, qo, ko, max_q, max_k, got["out"], got["lse"], g, got["grad_q"], got["grad_k"],
                                    got["grad_v"], **how)
    torch.cuda.synchronize()
    return got


def check(ctx, lq, lk, H, G, d, dt, how, seed=1, train=True, std=1.0, **kw):
    qo, ko = offsets(lq), offsets(lk)
    Q, K = int(qo[-1]), int(ko[-1])
    q, k, v = du.rand((Q, H, d), dt, seed, std), du.rand((K, G, d), dt, seed + 1, std), du.rand((K, G, d), dt, seed + 2)
    g = du.rand((Q, H, d), dt, seed + 3) if train else None
    how = dict(dict(scale=d ** -0.5), **how)
    ref = du.attention_ref(q, k, v, qo, ko, g=g, **how)
    got = run(ctx, q, k, v, qo, ko, how, g, **kw)
    for n, t in got.items():
        if n == "lse":
            none = ref[n][0] == -float("inf")
            assert torch.equal(t.cpu() == -float("inf"), none)
            du.within(t.cpu()[~none], ref[n][0][~none], ref[n][1][~none], what=n)
        else:
            du.within(t, *ref[n], what=n)
    return got


SLOPES = lambda H: 2.0 ** (-8.0 * torch.arange(1, H + 1) / H)  # noqa: E731


# lengths: none, one, edges of tiles of 32, 64 and 128 rows, several tiles
LENGTHS = {"small": [0, 1, 2, 31, 0, 32, 33, 5], "mid": [63, 1, 64, 65, 100], "long": [129, 300, 0, 7, 128], "one": [1],
           "none": [0, 0, 3, 0]}


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lens", list(LENGTHS))
@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(ctx, dt, lens, d, causal):
    check(ctx, LENGTHS[lens], LENGTHS[lens], 2, 2, d, dt, dict(causal=causal))


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("what", ["cap", "slopes", "prefix", "all", "all_not_causal"])
def test_caps_biases_and_prefixes(ctx, dt, what):
    lens = [70, 3, 0, 33, 150]
    prefix = torch.tensor([40, 0, 5, 200, 1], dtype=torch.int32)   # one longer than its list
    how = {"cap": dict(softcap=3.0, causal=True), "slopes": dict(slopes=SLOPES(4), causal=True),
           "prefix": dict(causal=True, prefix=prefix),
           "all": dict(softcap=3.0, slopes=SLOPES(4), causal=True, prefix=prefix),
           "all_not_causal": dict(softcap=3.0, slopes=SLOPES(4))}[what]
    check(ctx, lens, lens, 4, 2, 40, dt, how, std=2.0)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("H,G", [(1, 1), (6, 3), (8, 1), (5, 1), (12, 4)])
def test_shared_heads(ctx, dt, H, G):
    check(ctx, [20, 47, 1, 90], [20, 47, 1, 90], H, G, 24, dt, dict(causal=True, slopes=SLOPES(H)))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
def test_queries_and_keys_of_different_lengths(ctx, dt, causal):
    """More queries than keys leave the first ones of a causal list without any key; so do lists without keys."""
    lq, lk = [10, 50, 3, 0, 7, 200, 1, 40], [30, 20, 0, 9, 7, 65, 300, 39]
    prefix = torch.tensor([0, 0, 2, 1, 0, 3, 0, 100], dtype=torch.int32) if causal else None
    got = check(ctx, lq, lk, 4, 2, 32, dt, dict(causal=causal, prefix=prefix))
    if causal:
        assert not got["out"][10:40].any() and not got["grad_q"][10:40].any()   # 30 queries before the first key
        assert not got["out"][60:63].any()                                      # no keys at all


# keys are split over blocks where there are few tiles
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lk,H,G", [([700, 1, 0, 2100], 8, 2), ([5000], 1, 1), ([257, 512], 3, 3), ([4097], 20, 1)])
def test_one_query_per_list(ctx, dt, lk, H, G):
    check(ctx, [1] * len(lk), lk, H, G, 64, dt, dict(causal=True, softcap=5.0), train=False)
    check(ctx, [1] * len(lk), lk, H, G, 128, dt, dict(slopes=SLOPES(H)), train=False)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_splits_with_several_queries(ctx, dt):
    """Few tiles of longer queries: splits that lie behind a row's last key leave it alone."""
    check(ctx, [600, 40], [1300, 900], 2, 1, 32, dt, dict(causal=True), train=False)
    check(ctx, [900], [900], 1, 1, 16, dt, dict(causal=True, prefix=torch.tensor([300], dtype=torch.int32)), train=False)


def test_bounds_may_be_larger_than_the_lists(ctx):
    lens = [5, 60, 0, 33]
    a = check(ctx, lens, lens, 2, 2, 32, "bf16", dict(causal=True))
    b = check(ctx, lens, lens, 2, 2, 32, "bf16", dict(causal=True), max_q=5000, max_k=60_000)
    for n in ("out", "grad_q", "grad_k", "grad_v"):
        assert (a[n].float() - b[n].float()).norm() <= 0.02 * a[n].float().norm()


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_rows_apart_by_strides(ctx, dt):
    """Queries, keys and values in one array, gradients in another, and rows that are not neighbours."""
    lens, H, G, d = [33, 2, 100], 4, 2, 32
    o = offsets(lens)
    K = int(o[-1])
    both = du.rand((K, H + 2 * G, d), dt, 5).cuda()
    q, k, v = both[:, :H], both[:, H:H + G], both[:, H + G:]
    g = du.rand((K, H, d), dt, 6).cuda()
    how = dict(scale=0.2, causal=True)
    want = run(ctx, q.contiguous(), k.contiguous(), v.contiguous(), o, o, how, g)
    gb = torch.full((K, H + 2 * G, d), float("nan"), dtype=both.dtype, device="cuda")
    wide = torch.full((K, 3, H, d), 7.0, dtype=both.dtype, device="cuda")
    wide[:, 1] = q
    out, lse = torch.empty_like(want["out"]), torch.empty_like(want["lse"])
    oc = o.cuda()
    ctx.list_attention(wide[:, 1], k, v, oc, oc, 100, 100, out, lse, **how)
    ctx.list_attention_backward(wide[:, 1], k, v, oc, oc, 100, 100, out, lse, g, gb[:, :H], gb[:, H:H + G], gb[:, H + G:], **how)
    for got, n in ((out, "out"), (gb[:, :H], "grad_q"), (gb[:, H:H + G], "grad_k"), (gb[:, H + G:], "grad_v")):
        assert torch.equal(got, want[n]), n


@pytest.mark.parametrize("power", [-18, 6])
def test_fp16_gradients_of_any_size(ctx, power):
    """Gradients of the output that are far from 1 neither vanish nor overflow inside."""
    o = offsets([90, 40])
    q, k, v = (du.rand((130, 2, 64), "f16", s) for s in (1, 2, 3))
    g = (du.rand((130, 2, 64), "f16", 4).double() * 2.0 ** power).half()
    how = dict(scale=0.125, causal=True)
    ref = du.attention_ref(q, k, v, o, o, g=g, **how)
    got = run(ctx, q, k, v, o, o, how, g)
    for n in ("grad_q", "grad_k", "grad_v"):
        du.within(got[n], *ref[n], what=n)


def test_large_scores(ctx):
    """Scores of hundreds that rise along the keys move the running maximum at every tile."""
    o = offsets([300])
    q, k, v = (du.rand((300, 1, 32), "f32", s) for s in (1, 2, 3))
    q, k = q.abs(), k.abs() * torch.linspace(0.1, 40, 300)[:, None, None]
    how = dict(scale=0.5)
    ref = du.attention_ref(q, k, v, o, o, **how)
    got = run(ctx, q, k, v, o, o, how)
    du.within(got["out"], *ref["out"], what="out")
    du.within(got["lse"], *ref["lse"], what="lse")


def test_lists_do_not_touch_each_other(ctx):
    """A list of NaN and infinities leaves the lists around it as they are, forward and backward."""
    lens = [40, 17, 66]
    o = offsets(lens)
    q, k, v, g = (du.rand((123, 2, 32), "bf16", s) for s in (1, 2, 3, 4))
    how = dict(scale=0.3, causal=True)
    want = run(ctx, q, k, v, o, o, how, g)
    for t in (q, k, v, g):
        t[40:57] = float("nan")
        t[45] = float("inf")
    got = run(ctx, q, k, v, o, o, how, g)
    rows = torch.ones(123, dtype=torch.bool)
    rows[40:57] = False
    rows = rows.cuda()
    for n in want:
        assert torch.equal(got[n][rows], want[n][rows]), n


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("H,G,d", [(1, 1, 128), (4, 1, 24), (6, 3, 64)])
def test_many_splits(ctx, dt, H, G, d):
    """Single tokens whose keys are cut into more splits than a thread group goes through, an empty list and a short one."""
    check(ctx, [1, 1, 1, 0, 1], [9000, 0, 700, 5, 3], H, G, d, dt, dict(causal=True, softcap=3.0, slopes=SLOPES(H) / 64), train=False)


# lists of few rows (a wave to a tile); of single rows whose keys are divided; of tiles in phases; of whole groups
PLANTED = {"short": ([20, 45, 7], [20, 45, 7], 2, 2), "single": ([1, 3, 1], [700, 900, 300], 4, 2),
           "phases": ([150, 260, 40], [150, 260, 40], 2, 1), "groups": ([260] * 40, [260] * 40, 8, 4)}


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("name", list(PLANTED))
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("softcap", [0.0, 5.0])
def test_what_is_masked_may_hold_anything(ctx, dt, name, bad, softcap):
    """A key and a value that are not finite reach the rows that see them alone; so do a query and its gradient."""
    lq, lk, H, G = PLANTED[name]
    d = 128 if name == "groups" else 40
    qo, ko = offsets(lq), offsets(lk)
    Q, K = int(qo[-1]), int(ko[-1])
    q, k, v, g = du.rand((Q, H, d), dt, 1), du.rand((K, G, d), dt, 2), du.rand((K, G, d), dt, 3), du.rand((Q, H, d), dt, 4)
    how = dict(scale=d ** -0.5, causal=True, softcap=softcap)
    ref = du.attention_ref(q, k, v, qo, ko, g=g, **how)
    j = lk[1] - 2 if lq[1] < 5 else lk[1] // 2 + 3  # of the second list
    i = j - (lk[1] - lq[1])                          # the first query that sees it
    k1, v1 = k.clone(), v.clone()
    k1[int(ko[1]) + j, :, ::3] = bad
    v1[int(ko[1]) + j, :, 1::2] = bad
    got = run(ctx, q, k1, v1, qo, ko, how, g)
    rows = torch.ones(Q, dtype=torch.bool)
    rows[int(qo[1]) + i:int(qo[2])] = False
    for n in ("out", "grad_q"):
        du.within(got[n][rows.cuda()], ref[n][0][rows], ref[n][1][rows], what=n + " beside keys")
    du.within(got["lse"].cpu()[rows], ref["lse"][0][rows], ref["lse"][1][rows], what="lse beside keys")
    assert not got["out"][int(qo[1]) + i:int(qo[2]), :, 1::2].isfinite().any()
    q1, g1 = q.clone(), g.clone()
    q1[int(qo[1]) + i, :, ::3] = bad
    g1[int(qo[1]) + i, :, 1::2] = bad
    got = run(ctx, q1, k, v, qo, ko, how, g1)
    rows = torch.arange(Q) != int(qo[1]) + i
    keys = torch.ones(K, dtype=torch.bool)
    keys[int(ko[1]):int(ko[1]) + j + 1] = False
    for n, there in (("out", rows), ("grad_q", rows), ("grad_k", keys), ("grad_v", keys)):
        du.within(got[n][there.cuda()], ref[n][0][there], ref[n][1][there], what=n + " beside a query")
    assert not got["grad_v"][int(ko[1]):int(ko[1]) + j + 1, :, 1::2].isfinite().any()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("name", list(PLANTED))
def test_all_of_it_nan(ctx, dt, name):
    """Lists of NaN alone: NaN in every row, in time."""
    lq, lk, H, G = PLANTED[name]
    nan = torch.full((1, 1, 64), float("nan"), dtype=du.rand((1,), dt, 1).dtype)
    q, k = nan.expand(sum(lq), H, 64).contiguous(), nan.expand(sum(lk), G, 64).contiguous()
    got = run(ctx, q, k, k.clone(), offsets(lq), offsets(lk), dict(scale=0.1, causal=True), q.clone())
    for n, t in got.items():
        assert t.isnan().all(), n


def test_rows_too_far_apart_are_refused(ctx):
    """Rows of 16 MiB and more from one to the next: offsets inside a tile are held in 32 bits."""
    from paper_2211_05239_amd import recd
    q = torch.zeros(3, 1, 16, device="cuda")
    o = torch.tensor([0, 3], device="cuda")
    wide = torch.empty_strided((3, 1, 16), (1 << 22, 16, 1), device="cuda")
    for a in ((wide, q, q), (q, wide, q), (q, q, wide)):
        with pytest.raises(recd.RecdError):
            ctx.list_attention(*a, o, o, 3, 3, torch.empty_like(q), scale=1.0)
    ctx.list_attention(q, q, q, o, o, 3, 3, torch.empty_like(q), scale=1.0)


def test_same_bits_again(ctx):
    lens = [300, 5, 0, 77, 129]
    a = check(ctx, lens, lens, 4, 2, 64, "bf16", dict(causal=True, softcap=4.0))
    b = check(ctx, lens, lens, 4, 2, 64, "bf16", dict(causal=True, softcap=4.0))
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_gradients_against_differences(ctx):
    """Central differences of sum(g * out) in fp32: off by the outputs' rounding over the step and its square."""
    lq, lk = [3, 2], [4, 3]
    qo, ko = offsets(lq), offsets(lk)
    q, k, v, g = (du.rand(s, "f32", i) for i, s in enumerate(((5, 2, 4), (7, 1, 4), (7, 1, 4), (5, 2, 4))))
    how = dict(scale=0.6, softcap=2.0, slopes=SLOPES(2), causal=True, prefix=torch.tensor([1, 0], dtype=torch.int32))
    got = run(ctx, q, k, v, qo, ko, how, g)
    h = 2.0 ** -7

    def value():
        return float((run(ctx, q, k, v, qo, ko, how)["out"].double().cpu() * g.double()).sum())

    for name, t in (("grad_q", q), ("grad_k", k), ("grad_v", v)):
        flat = t.view(-1)
        for i in range(flat.numel()):
            old = float(flat[i])
            flat[i] = old + h
            up = value()
            flat[i] = old - h
            down = value()
            flat[i] = old
            assert abs((up - down) / (2 * h) - float(got[name].view(-1)[i])) < 2e-3, (name, i)


def test_a_cache_beyond_2_to_31_elements(ctx):
    """Keys and values whose positions pass 32 bits: rows 16 K elements apart, the second list behind 2^31."""
    rows, wide, d = 150_000, 16_384, 64
    cache = torch.empty(rows, wide // d, d, dtype=torch.float16, device="cuda")
    k, v = cache[:, :2], cache[:, -2:]
    n = [rows - 700, 700]
    o = offsets(n)
    kc, vc = du.rand((rows, 2, d), "f16", 1, 0.5), du.rand((rows, 2, d), "f16", 2)
    k.copy_(kc.cuda())
    v.copy_(vc.cuda())
    q = du.rand((2, 4, d), "f16", 3)
    qo = offsets([1, 1])
    how = dict(scale=0.125, causal=True)
    ref = du.attention_ref(q, kc, vc, qo, o, **how)
    out = torch.empty(2, 4, d, dtype=torch.float16, device="cuda")
    ctx.list_attention(q.cuda(), k, v, qo.cuda(), o.cuda(), 1, rows, out, **how)
    du.within(out, *ref["out"], what="out")


def test_another_stream_and_a_graph(ctx):
    from paper_2211_05239_amd import recd
    lens = [90, 3, 0, 200]
    o = offsets(lens).cuda()
    q, k, v, g = (du.rand((293, 2, 32), "f16", s).cuda() for s in (1, 2, 3, 4))
    how = dict(scale=0.3, causal=True)
    want = run(ctx, q, k, v, o, o, how, g)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c = recd.Context(0)
        got = {n: torch.zeros_like(t) for n, t in want.items()}

        def step():
            c.list_attention(q, k, v, o, o, 200, 200, got["out"], got["lse"], **how)
            c.list_attention_backward(q, k, v, o, o, 200, 200, got["out"], got["lse"], g, got["grad_q"], got["grad_k"],
                                      got["grad_v"], **how)

        step()
        s.synchronize()
        for n in want:
            assert torch.equal(got[n], want[n]), n
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
        for i in range(4):
            for t in got.values():
                t.fill_(float("nan"))
            graph.replay()
            s.synchronize()
            for n in want:
                assert torch.equal(got[n], want[n]), (i, n)
            run(c, q, k, v, o, o, how, g)
        c.close()


def test_validation(ctx):
    from paper_2211_05239_amd import recd
    q = du.rand((10, 1, 16), "f32", 1)
    ctx.set_option(recd.RECD_OPT_VALIDATE, 1)
    try:
        run(ctx, q, q, q, offsets([4, 6]), offsets([4, 6]), dict(scale=1.0), q)
        for bad, most in ((torch.tensor([0, 11, 10]), 11), (torch.tensor([1, 4, 10]), 10), (torch.tensor([0, 4, 9]), 10),
                          (offsets([4, 6]), 5)):
            with pytest.raises(recd.RecdError) as e:
                run(ctx, q, q, q, bad, bad, dict(scale=1.0), q, max_q=most, max_k=most)
            assert e.value.status == recd.RECD_EBOUNDS
    finally:
        ctx.set_option(recd.RECD_OPT_VALIDATE, 0)


def test_refusals(ctx):
    import ctypes as C

    from paper_2211_05239_amd import recd
    lib, h = recd._lib, ctx._h
    buf = torch.zeros(4096, device="cuda")
    p = buf.data_ptr()
    good = dict(heads=2, kv_heads=2, head_dim=16, dtype=0, lists=1, max_q=4, max_k=4, q_rows=4, k_rows=4, q_offsets=p,
                k_offsets=p, q_stride=32, k_stride=32, v_stride=32, scale=1.0, softcap=0.0, slopes=None, prefix=None, causal=1)

    def forward(ctx_=h, q=p, k=p, v=p, out=p, **kw):
        a = recd._Attention(**dict(good, **kw))
        return lib.recd_list_attention(ctx_, C.byref(a), q, k, v, out, None)

    def backward(out=p, lse=p, g=p, gq=p, gk=p, gv=p, s=(32, 32, 32), **kw):
        a = recd._Attention(**dict(good, **kw))
        return lib.recd_list_attention_backward(h, C.byref(a), p, p, p, out, lse, g, gq, gk, gv, *s)

    bad = recd.RECD_EINVAL
    for kw in (dict(ctx_=None), dict(heads=0), dict(heads=3), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=6),
               dict(head_dim=132, q_stride=1000, k_stride=1000, v_stride=1000), dict(head_dim=12, dtype=1), dict(dtype=3),
               dict(lists=-1), dict(max_q=-1), dict(max_k=-1), dict(q_rows=-1), dict(k_rows=-1), dict(lists=0),
               dict(q_offsets=None), dict(k_offsets=None), dict(q_stride=28), dict(k_stride=16), dict(v_stride=31),
               dict(q_stride=34), dict(softcap=-1.0), dict(softcap=float("nan")), dict(softcap=float("inf")),
               dict(prefix=p, causal=0), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q=p + 4),
               dict(out=p + 4), dict(max_q=1 << 31), dict(lists=1 << 31)):
        assert forward(**kw) == bad, kw
    for kw in (dict(out=None), dict(lse=None), dict(g=None), dict(gq=None), dict(gk=None), dict(gv=None), dict(gk=p + 8),
               dict(s=(28, 32, 32)), dict(s=(32, 16, 32)), dict(s=(32, 32, 33)), dict(head_dim=6)):
        assert backward(**kw) == bad, kw
    assert lib.recd_list_attention(h, None, p, p, p, p, None) == bad
    assert forward(lists=0, q_rows=0, k_rows=0, q_offsets=None, k_offsets=None, q=None, k=None, v=None, out=None) == recd.RECD_OK


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("name", list(PLANTED))
def test_an_infinity_that_is_seen_beside_a_nan_that_is_not(ctx, dt, name):
    """A row that sees an infinite value gives that infinity, whatever lies in the places behind its last key."""
    lq, lk, H, G = PLANTED[name]
    d = 128 if name == "groups" else 40
    qo, ko = offsets(lq), offsets(lk)
    Q, K = int(qo[-1]), int(ko[-1])
    q, k, v = du.rand((Q, H, d), dt, 1), du.rand((K, G, d), dt, 2), du.rand((K, G, d), dt, 3)
    j = lk[1] - 2 if lq[1] < 5 else lk[1] // 2 + 3   # the infinity's key of the second list; behind it the NaN's
    i = int(qo[1]) + j - (lk[1] - lq[1])             # the one query that sees the first and not the second
    v[int(ko[1]) + j, :, 0] = float("inf")
    v[int(ko[1]) + j, :, 1] = -float("inf")
    v[int(ko[1]) + j + 1] = float("nan")
    got = run(ctx, q, k, v, qo, ko, dict(scale=d ** -0.5, causal=True))
    out = got["out"].cpu().double()
    assert (out[i, :, 0] == float("inf")).all() and (out[i, :, 1] == -float("inf")).all() and out[i, :, 2:].isfinite().all()
    assert out[i + 1:int(qo[2])].isnan().all()
    rows = torch.ones(Q, dtype=torch.bool)
    rows[i:int(qo[2])] = False
    assert out[rows].isfinite().all()


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_values_gradients_beside_an_infinite_output(ctx, dt):
    """A last query whose output is infinite where its gradient is zero (so g . out is a NaN) hides no other row's NaN."""
    n, d = 70, 32
    o = offsets([n])
    q, k, v, g = (du.rand((n, 1, d), dt, s) for s in (1, 2, 3, 4))
    how = dict(scale=0.2, causal=True)
    v[n - 1, 0, 0] = float("inf")          # the last query alone sees it
    g[n - 1, 0, 0] = 0.0
    g[40] = float("nan")
    want = du.attention_ref(q, k, torch.nan_to_num(v, posinf=1.0), o, o, g=torch.nan_to_num(g), **how)
    got = run(ctx, q, k, v, o, o, how, g)
    assert got["grad_v"][:41].isnan().all()
    du.within(got["grad_v"][41:], want["grad_v"][0][41:], want["grad_v"][1][41:], what="grad_v")


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("where", ["gradient", "value", "everywhere"])
def test_an_overflow_costs_a_few_passes(ctx, dt, where):
    """One infinity in a long list's gradient or values, as after an overflow, or all of them: no more than a few times as long."""
    n, H, G, d = 2048, 4, 2, 128
    o = offsets([n]).cuda()
    q, g = du.rand((n, H, d), dt, 1).cuda(), du.rand((n, H, d), dt, 4).cuda()
    k, v = du.rand((n, G, d), dt, 2).cuda(), du.rand((n, G, d), dt, 3).cuda()
    out, lse, gq, gk, gv = torch.empty_like(q), torch.empty(n, H, device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)

    def took():
        best = 1e9
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            torch.cuda.synchronize()
            a.record()
            ctx.list_attention(q, k, v, o, o, n, n, out, lse, scale=0.1, causal=True)
            ctx.list_attention_backward(q, k, v, o, o, n, n, out, lse, g, gq, gk, gv, scale=0.1, causal=True)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b))
        return best

    clean = took()
    if where == "gradient":
        g[1200, 1, 5] = float("inf")
    elif where == "value":
        v[700, 1, 5] = float("inf")
    else:
        g[:] = float("inf")
    assert took() < 6 * clean + 0.2


def scaled_rows(x, rows, by):
    y = x.clone()
    y[rows] = (y[rows].double() * by).to(y.dtype)
    return y


# (a wave to a tile, phases, groups)
@pytest.mark.parametrize("lens,H,G,d", [([20, 45, 7], 2, 1, 32), ([150, 260, 40], 2, 1, 64), ([260] * 24, 8, 4, 128)])
@pytest.mark.parametrize("where", ["both", "apart"])
def test_fp16_gradients_of_lists_beside_much_larger_ones(ctx, lens, H, G, d, where):
    """Values and gradients of one list (or of two) that are thousands of times as large leave the others' bits alone: each
    list is held to the bound of its own data."""
    o = offsets(lens)
    K = int(o[-1])
    q, k, v, g = du.rand((K, H, d), "f16", 1), du.rand((K, G, d), "f16", 2), du.rand((K, G, d), "f16", 3), du.rand((K, H, d), "f16", 4)
    how = dict(scale=d ** -0.5, causal=True)
    large = [1] if where == "both" else [0, 1]
    v = scaled_rows(v, slice(int(o[1]), int(o[2])), 4000.0)
    g = scaled_rows(g, slice(int(o[large[0]]), int(o[large[0] + 1])), 4000.0)
    got = run(ctx, q, k, v, o, o, how, g)
    for l in [l for l in range(len(lens)) if l != 1][:3]:
        a, b = int(o[l]), int(o[l + 1])
        ref = du.attention_ref(q[a:b], k[a:b], v[a:b], offsets([b - a]), offsets([b - a]), g=g[a:b], **how)
        for n in ("grad_q", "grad_k", "grad_v"):
            du.within(got[n][a:b], *ref[n], what=f"{n} of list {l}")


@pytest.mark.parametrize("n,H,G,d", [(45, 2, 1, 32), (260, 2, 1, 64), (512, 1, 1, 128)])
def test_fp16_gradients_before_a_large_last_row(ctx, n, H, G, d):
    """Rows that do not see the last key keep the bits of their gradients, however large its value."""
    o = offsets([n])
    q, k, v, g = du.rand((n, H, d), "f16", 1), du.rand((n, G, d), "f16", 2), du.rand((n, G, d), "f16", 3), du.rand((n, H, d), "f16", 4)
    how = dict(scale=d ** -0.5, causal=True)
    ref = du.attention_ref(q[:-1], k[:-1], v[:-1], offsets([n - 1]), offsets([n - 1]), g=g[:-1], **how)
    got = run(ctx, q, k, scaled_rows(v, slice(n - 1, n), 10_000.0), o, o, how, scaled_rows(g, slice(n - 1, n), 10_000.0))
    du.within(got["grad_q"][:-1], *ref["grad_q"], what="grad_q")


def test_fp16_gradients_of_rows_that_rise(ctx):
    """Weights that grow along a list by 2^30 in all, small ones first and small ones last."""
    n, d = 300, 64
    o = offsets([n])
    q, k, v = (du.rand((n, 1, d), "f16", s, 0.5) for s in (1, 2, 3))
    how = dict(scale=0.125)
    for up in (True, False):
        size = 2.0 ** torch.linspace(-22, 8, n, dtype=torch.float64)
        size = size if up else size.flip(0)
        g = (du.rand((n, 1, d), "f16", 4).double() * size[:, None, None]).half()
        ref = du.attention_ref(q, k, v, o, o, g=g, **how)
        got = run(ctx, q, k, v, o, o, how, g)
        for name in ("grad_q", "grad_k", "grad_v"):
            du.within(got[name], *ref[name], what=name)
        some = (g.double().abs().sum((1, 2)) > 0) & (size > 2.0 ** -10)
        off = (got["grad_q"].double().cpu() - ref["grad_q"][0])[some].norm(dim=(1, 2)) / ref["grad_q"][0][some].norm(dim=(1, 2))
        assert off.max() < 0.02      # every row to its own size (2^-11 in the operands, the output stored in 16 bits)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("name", list(PLANTED))
@pytest.mark.parametrize("d,softcap", [(24, 0.0), (40, 0.0), (40, 5.0), (80, 0.0)])
def test_an_infinite_last_element_of_a_head(ctx, dt, name, d, softcap):
    """A key whose last elements are infinite, against queries that are positive there, scores -inf (capped: -cap), however
    much wider than the head a tile is: it has no weight, and no part in the others' gradients."""
    lq, lk, H, G = PLANTED[name]
    if name == "groups" and d != 80:
        H, G = 4, 4
    qo, ko = offsets(lq), offsets(lk)
    Q, K = int(qo[-1]), int(ko[-1])
    q, k, v, g = du.rand((Q, H, d), dt, 1), du.rand((K, G, d), dt, 2), du.rand((K, G, d), dt, 3), du.rand((Q, H, d), dt, 4)
    j = int(ko[1]) + lk[1] // 2
    q[..., -3:] = q[..., -3:].abs() + 0.1
    k[j, :, -3:] = -float("inf")
    got = run(ctx, q, k, v, qo, ko, dict(scale=d ** -0.5, softcap=softcap), g)
    fine = k.clone()
    fine[j, :, -3:] = -1000.0 if dt != "f32" else -1e6   # next to no weight
    ref = du.attention_ref(q, fine, v, qo, ko, scale=d ** -0.5, softcap=softcap, g=g)
    for n in ("out", "lse"):
        du.within(got[n], *ref[n], what=n)
    if not softcap:      # (the stand-in's weight is 1e-14 and less, the infinity's none)
        assert not got["grad_k"][j].any() and not got["grad_v"][j].any()
    others = torch.ones(K, dtype=torch.bool)
    others[j] = False
    for n in ("grad_k", "grad_v"):
        du.within(got[n][others.cuda()], ref[n][0][others], ref[n][1][others], what=n)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("name", list(PLANTED))
def test_a_cap_far_above_the_scores_changes_nothing(ctx, dt, name):
    """cap * tanh(z / cap) is z where cap is large (by z^3 / 3 cap^2, 1e-11 here): no accuracy goes with the cap's size."""
    lq, lk, H, G = PLANTED[name]
    d = 64
    qo, ko = offsets(lq), offsets(lk)
    q, k, v, g = (du.rand((n, h, d), dt, s) for s, (n, h) in enumerate(((int(qo[-1]), H), (int(ko[-1]), G), (int(ko[-1]), G), (int(qo[-1]), H))))
    how = dict(scale=d ** -0.5, causal=True)
    ref = du.attention_ref(q, k, v, qo, ko, g=g, **how)
    got = run(ctx, q, k, v, qo, ko, dict(how, softcap=2.0 ** 22), g)
    for n, t in got.items():
        du.within(t, *ref[n], what=n)


@pytest.mark.parametrize("causal", [False, True])
def test_distances_beyond_2_to_24(ctx, causal):
    """Positions that fp32 does not hold: the last queries of a list of 2^24 + 101 rows see their neighbours at exact distances."""
    n, tail, d = 2 ** 24 + 101, 400, 8
    k, v = (torch.zeros(n, 1, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kt, vt = du.rand((tail, 1, d), "bf16", 1), du.rand((tail, 1, d), "bf16", 2)
    k[-tail:], v[-tail:] = kt.cuda(), vt.cuda()
    q, g = du.rand((5, 1, d), "bf16", 3), du.rand((5, 1, d), "bf16", 4)
    how = dict(scale=0.3, slopes=torch.tensor([0.5]), causal=causal)
    ref = du.attention_ref(q, kt, vt, offsets([5]), offsets([tail]), g=g, **how)   # (beyond the tail exp(-200))
    got = run(ctx, q, k, v, offsets([5]), offsets([n]), how, g)
    for name in ("out", "lse", "grad_q"):
        du.within(got[name], *ref[name], what=name)
    for name in ("grad_k", "grad_v"):
        du.within(got[name][-tail:], *ref[name], what=name)


def test_lengths_and_tiles_beyond_a_launch_are_refused(ctx):
    """By the descriptor alone, before anything is launched or read."""
    import ctypes as C

    from paper_2211_05239_amd import recd
    buf = torch.zeros(4096, device="cuda")
    p = buf.data_ptr()
    good = dict(heads=4, kv_heads=4, head_dim=16, dtype=0, lists=1, max_q=4, max_k=4, q_rows=4, k_rows=4, q_offsets=p,
                k_offsets=p, q_stride=64, k_stride=64, v_stride=64, scale=1.0, softcap=0.0, slopes=None, prefix=None, causal=1)
    most = (1 << 31) - (1 << 18)
    many = dict(lists=1 << 27, q_rows=1 << 27, k_rows=1 << 27, max_q=3, max_k=3)
    for kw in (dict(max_k=most + 1, k_rows=most + 1), dict(max_q=most // 4 + 1, q_rows=most // 4 + 1), many,
               dict(many, lists=1 << 25, q_rows=1 << 25, k_rows=1 << 25, heads=32, kv_heads=32, q_stride=512, k_stride=512, v_stride=512)):
        a = recd._Attention(**dict(good, **kw))
        s = (a.q_stride, a.k_stride, a.v_stride)
        assert recd._lib.recd_list_attention_backward(ctx._h, C.byref(a), p, p, p, p, p, p, p, p, p, *s) == recd.RECD_EINVAL, kw
        if a.kv_heads == 4:   # (the forward pass of many short lists goes through several heads in a block)
            assert recd._lib.recd_list_attention(ctx._h, C.byref(a), p, p, p, p, None) == recd.RECD_EINVAL, kw


# (a wave to a list: all its keys in one tile, and in several; phases; groups)
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("lens,H,G,d", [([20, 31, 7], 2, 2, 32), ([60, 100], 1, 1, 64), ([150, 260], 2, 1, 64), ([300] * 20, 8, 4, 128)])
@pytest.mark.parametrize("softcap,copies", [(0.0, False), (60.0, False), (0.0, True)])
def test_gradients_of_rows_that_one_key_takes(ctx, dt, lens, H, G, d, softcap, copies):
    """Rows whose weight lies on one key (or on two that are the same, with the same value): what is left, p_j (dp_j - delta), keeps
    its accuracy though dp and delta are nearly equal there and delta is at first taken from the rounded output.

    With e what that delta is off by, u a rounding to the type, eta what fp32 leaves of a probability and tau of dp: weights
    are rounded, u (|ds| + p |e|); the sum of p (dp - delta) gives e back but for eta and tau, exactly for the gradients by keys; in those
    by queries e remains beside the heaviest key's k* alone, as e (sum p k - k*)."""
    o = offsets(lens)
    K = int(o[-1])
    gen = torch.Generator().manual_seed(5)
    k, v, g = du.rand((K, G, d), dt, 2), du.rand((K, G, d), dt, 3), du.rand((K, H, d), dt, 4)
    q = torch.empty(K, H, d, dtype=k.dtype)
    for a, b in zip(o[:-1].tolist(), o[1:].tolist()):
        if copies:
            half = (b - a) // 2
            k[a + half:a + 2 * half], v[a + half:a + 2 * half] = k[a:a + half], v[a:a + half]
        for h in range(H):
            keys = k[a:b, h // (H // G)].double()
            to = keys[torch.randperm(b - a, generator=gen)]
            z = torch.linspace(2.0, 25.0, b - a, dtype=torch.float64)[torch.randperm(b - a, generator=gen)][:, None]
            q[a:b, h] = (to * z / to.square().sum(1, keepdim=True)).to(q.dtype)
    got = {n: t.double().cpu() for n, t in run(ctx, q, k, v, o, o, dict(scale=1.0, softcap=softcap), g).items()}
    u, E, peaked = du.U[q.dtype], du.E, 0
    tiny = 2.0 ** -25 if dt == "f16" else 0.0
    for a, b in zip(o[:-1].tolist(), o[1:].tolist()):
        for G_ in range(G):
            ks, vs = k[a:b, G_].double(), v[a:b, G_].double()
            gk, gk_off = torch.zeros_like(ks), torch.zeros(b - a, dtype=torch.float64)
            for h in range(G_ * (H // G), (G_ + 1) * (H // G)):
                qs, gs = q[a:b, h].double(), g[a:b, h].double()
                s = qs @ ks.t()
                t = torch.tanh(s / softcap) if softcap else torch.zeros_like(s)
                z, bend = (softcap * t if softcap else s), 1 - t * t
                p = torch.softmax(z, 1)
                dp = gs @ vs.t()
                delta = (p * dp).sum(1, keepdim=True)
                out = p @ vs
                ds = p * bend * (dp - delta)
                dz = 2 * E * (d / 16 + 4) * (qs.abs() @ ks.abs().t()) + 8 * E * (z.abs() + torch.logsumexp(z, 1)[:, None].abs() + softcap)
                eta = 4 * dz.max(1, keepdim=True).values + 16 * E
                tau = 4 * E * (d + 8) * (gs.abs() @ vs.abs().t()).max(1, keepdim=True).values
                e = (gs.abs() * (u * out.abs() + (u + 2 * eta) * (p @ vs.abs()))).sum(1, keepdim=True) + tau
                left = eta * (p * (dp - delta).abs()).sum(1, keepdim=True) + tau + eta * e   # of delta, once settled
                kn, big = ks.norm(dim=1), ks.norm(dim=1).max()
                top = p.argmax(1)
                apart = ((p * bend) @ ks - bend.gather(1, top[:, None]) * ks[top]).norm(dim=1)
                want = ds @ ks
                fp32 = (p * (eta * (dp - delta).abs() + tau)) @ kn + (left * big)[:, 0] * 2
                bound = u * want.norm(dim=1) + u * (ds.abs() + p * e) @ kn + e[:, 0] * apart + fp32 \
                    + tiny * (b - a) * (ds.abs().max(1).values + e[:, 0]) * big
                off = (got["grad_q"][a:b, h] - want).norm(dim=1)
                assert (off <= bound).all(), float((off / bound).max())
                peaked += int(((1 - p.max(1).values) < 1e-3).sum())
                gk += ds.t() @ qs
                qn = qs.norm(dim=1)
                gk_off += u * ds.abs().t() @ qn + (p * (eta * (dp - delta).abs() + tau + left)).t() @ qn \
                    + tiny * (b - a) * ds.abs().max(0).values * qn.max()
            off = (got["grad_k"][a:b, G_] - gk).norm(dim=1)
            bound = u * gk.norm(dim=1) + gk_off
            assert (off <= bound).all(), float((off / bound).max())
    assert copies or peaked > 5
