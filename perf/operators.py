"""The dense operators that run on the rows of deduplicated lists, as cases to be measured.

A sequence feature's lists are looked up unpooled, once per unique list, into rows [M, D] with offsets.  Three
operators work on such rows:

  norm       layer norm of every row; its gradients, with those of the weight and the bias summed over all rows
  attention  attention inside every list (no row sees another list): queries and keys by offsets of their own, grouped
             heads, scores capped by a tanh, a bias that falls with the distance, causal with a prefix that all queries
             see; its gradients; one new query row per list for serving
  loss       softmax cross entropy of every row against a whole embedding table as the vocabulary; its gradients by
             the rows and by the table

Lengths follow a law's quantiles, in an order drawn from the seed, so every seed has the same amount of work.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-5
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def _norm(name, dtype, n, D, train):
    return {"name": name, "kind": "norm", "dtype": dtype, "n": n, "D": D, "train": train}


def _attention(name, dtype, lists, law, k_max, queries, heads, kv_heads, head_dim, causal, softcap, slopes, prefix, packed,
               train):
    """queries: "same" (a list's rows are its queries too), "one" (one row per list) or "other" (another length)."""
    return {"name": name, "kind": "attention", "dtype": dtype, "lists": lists, "law": law, "k_max": k_max,
            "queries": queries, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "causal": causal,
            "softcap": softcap, "slopes": slopes, "prefix": prefix, "packed": packed, "train": train}


def _loss(name, dtype, n, rows, D, ignored, train):
    return {"name": name, "kind": "loss", "dtype": dtype, "n": n, "rows": rows, "D": D, "ignored": ignored,
            "train": train}


def listed():
    return [
        # the rows of one request's unique lists, to be scored: launches count
        _norm("norm_request_f16", "f16", 37, 32, False),
        # the unique ids of a training batch (benchmark configuration 2: 16 features, 512 sessions), both directions
        _norm("norm_train_bf16", "bf16", 300_007, 128, True),
        # wide fp32 rows, an odd number of pieces per row
        _norm("norm_train_wide_f32", "f32", 50_021, 516, True),
        # a request's last positions scored against a table of 100 K rows (configuration 1's table), no gradient
        _loss("loss_request_f32", "f32", 37, 100_000, 64, 0.0, False),
        # training on fp32 tables of that size, some rows without a target
        _loss("loss_train_f32", "f32", 1500, 100_000, 64, 0.1, True),
        # training on an odd table in 16 bits, rows of twelve pieces
        _loss("loss_train_ragged_f16", "f16", 2500, 300_007, 96, 0.05, True),
        # the largest: a table of a million rows of 128 (configurations 2 to 5)
        _loss("loss_train_bf16", "bf16", 4096, 1_000_000, 128, 0.05, True),
        # one new token of each of 37 histories of up to 16 K rows: serving, grouped heads, capped scores
        _attention("token_f16", "f16", 37, "uniform", 16_384, "one", 8, 2, 64, True, 30.0, False, False, False, False),
        # a training batch of short lists (configuration 2's lengths), projections packed in one array
        _attention("short_lists_bf16", "bf16", 8192, "zipf", 100, "same", 4, 4, 32, True, 0.0, True, False, True, True),
        # fp32 training, lists of up to 500 rows, odd head size, queries of other lengths than the keys
        _attention("ragged_f32", "f32", 61, "uniform", 500, "other", 6, 3, 24, True, 0.0, True, True, False, True),
        # evaluation of long histories, grouped heads, no causal mask
        _attention("histories_f16", "f16", 24, "uniform", 2048, "same", 8, 2, 64, False, 50.0, False, False, False, False),
        # the longest: histories of up to 4096 rows, training with all the masks and biases at once
        _attention("long_bf16", "bf16", 8, "uniform", 4096, "same", 8, 4, 128, True, 30.0, True, True, True, True),
    ]


def draw(rng):
    """One more case of the same ranges: no larger than the largest listed one of its kind."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["norm", "attention", "attention", "loss"])
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    train = rng.random() < 0.6
    per = 4 if dtype == "f32" else 8   # values of a 16-byte piece
    if kind == "norm":
        D = per * log(4, 200)
        c = _norm("", dtype, min(log(1, 400_000), 40_000_000 // D), D, train)
    elif kind == "loss":
        D = min(256, per * log(3, 64))
        rows = log(20_000, 1_000_000)
        most = 4e9 / rows if dtype != "f32" else 3e8 / rows
        c = _loss("", dtype, max(1, min(log(1, 8192), int(most * min(1, 128 / D)))), rows, D, rng.choice([0.0, 0.1, 0.5]), train)
    else:
        c = _draw_attention(rng, log, dtype, train)
    del c["name"]
    return c


def _draw_attention(rng, log, dtype, train):
    head_dim = rng.choice([16, 24, 32, 40, 64, 64, 80, 128, 128])
    kv_heads = rng.choice([1, 2, 3, 4])
    heads = min(8, kv_heads * rng.choice([1, 2, 4]) if kv_heads < 3 else kv_heads * rng.choice([1, 2]))
    queries = rng.choice(["same", "same", "same", "one", "other"]) if not train else rng.choice(["same", "same", "other"])
    k_max = log(8, 16_384 if queries == "one" else 4096)
    causal = rng.random() < 0.7
    # at most as many pairs as the longest case, in no more room than the card has for the padded form
    pairs = k_max * (1 if queries == "one" else k_max) * heads
    most = (1.0e9 if dtype != "f32" else 1.0e8) / pairs
    rows_most = 4e7 / (k_max * heads * head_dim)
    lists = max(1, min(log(1, 8192), int(most), int(rows_most)))
    packed = queries == "same" and heads == kv_heads and rng.random() < 0.5
    return _attention("", dtype, lists, rng.choice(["uniform", "zipf", "even"]), k_max, queries, heads, kv_heads,
                      head_dim, causal, rng.choice([0.0, 0.0, 20.0, 50.0]), rng.random() < 0.5, causal and rng.random() < 0.4,
                      packed, train)


# ---- inputs --------------------------------------------------------------------------------------------------

def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * int(seed) + tag)
    return g


def _normal(seed, tag, shape, dtype, std=1.0, mean=0.0):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(mean, std, generator=_gen(seed, tag))


def _quantiles(law, n, most):
    """n lengths of at most `most`, ascending."""
    q = (np.arange(n) + 0.5) / n
    if law == "even":
        return np.full(n, most, dtype=np.int64)
    if law == "uniform":
        return np.minimum(most, np.floor(q * (most + 1)).astype(np.int64))
    p = np.arange(1, most + 1, dtype=np.float64) ** -1.2
    c = np.cumsum(p)
    return np.minimum(most - 1, np.searchsorted(c, q * c[-1], side="right")).astype(np.int64) + 1


def _lengths(c):
    """(query rows, key rows) of every list, in the law's order."""
    k = _quantiles(c["law"], c["lists"], c["k_max"])
    if c["queries"] == "one":
        return np.ones_like(k), k
    if c["queries"] == "same":
        return k, k
    # from none to a few more than the keys, which a causal mask then leaves without any
    i = np.arange(len(k))
    return (k * ((i + 2) % 5) // 4 + (i + 1) % 4).astype(np.int64), k


def _prefixes(c, k):
    return (k // 3 * (np.arange(len(k)) % 3)).astype(np.int32)


def prepare(case, seed):
    c, dt = case, DTYPE[case["dtype"]]
    if c["kind"] == "norm":
        n, D = c["n"], c["D"]
        s = {"case": c, "x": _normal(seed, 3, (n, D), dt, 1.5, 0.3), "weight": _normal(seed, 5, (D,), torch.float32, 0.2, 1.0),
             "bias": _normal(seed, 7, (D,), torch.float32, 0.2)}
        s["y"] = torch.empty_like(s["x"])
        if c["train"]:
            s.update(grad_y=_normal(seed, 11, (n, D), dt), stats=torch.empty(n, 2, device=DEV), grad_x=torch.empty_like(s["x"]),
                     grad_weight=torch.empty(D, device=DEV), grad_bias=torch.empty(D, device=DEV))
        return s
    if c["kind"] == "loss":
        n, V, D = c["n"], c["rows"], c["D"]
        # rows behind a layer norm, a table whose logits spread by about two
        s = {"case": c, "x": _normal(seed, 13, (n, D), dt), "table": _normal(seed, 17, (V, D), dt, 2.0 / math.sqrt(D)),
             "scale": 1.0}
        u = torch.rand(n, generator=_gen(seed, 19), device=DEV, dtype=torch.float64)
        skewed = (V ** u - 1).to(torch.int64).clamp_(0, V - 1)            # about 1/k, as ids are
        none = torch.rand(n, generator=_gen(seed, 23), device=DEV) < c["ignored"]
        s["targets"] = torch.where(none, -1, (skewed * 7919) % V)
        s["loss"], s["lse"] = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        if c["train"]:
            # the weight of every row in the batch's loss; fp16 gradients are scaled up, as they are in training
            s["grad_loss"] = torch.rand(n, generator=_gen(seed, 29), device=DEV) + 0.5
            s["grad_loss"] *= 64.0 if c["dtype"] == "f16" else 1.0 / n
            s.update(mean_row=torch.empty(n, D, device=DEV), grad_x=torch.empty_like(s["x"]), grad_table=torch.empty_like(s["table"]))
        return s
    rng = np.random.default_rng(1_000_003 * int(seed) + 31)
    order = rng.permutation(c["lists"])
    nq, nk = (x[order] for x in _lengths(c))
    H, G, d = c["heads"], c["kv_heads"], c["head_dim"]

    def offsets(n):
        return torch.from_numpy(np.concatenate([[0], np.cumsum(n)])).to(DEV)

    s = {"case": c, "q_offsets": offsets(nq), "max_q": int(nq.max()), "max_k": int(nk.max())}
    s["k_offsets"] = s["q_offsets"] if c["queries"] == "same" else offsets(nk)
    Q, K = int(nq.sum()), int(nk.sum())
    if c["packed"]:
        both = _normal(seed, 37, (K, H + 2 * G, d), dt)
        s["q"], s["k"], s["v"] = both[:, :H], both[:, H:H + G], both[:, H + G:]
    else:
        s["q"], s["k"], s["v"] = _normal(seed, 37, (Q, H, d), dt), _normal(seed, 41, (K, G, d), dt), _normal(seed, 43, (K, G, d), dt)
    s["scale"] = 1.5 / math.sqrt(d)
    s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, H + 1, device=DEV, dtype=torch.float32) / H) if c["slopes"] else None
    s["prefix"] = torch.from_numpy(_prefixes(c, _lengths(c)[1])[order]).to(DEV) if c["prefix"] else None
    s["out"] = torch.empty(Q, H, d, dtype=dt, device=DEV)
    s["lse"] = torch.empty(Q, H, device=DEV) if c["train"] else None
    if c["train"]:
        s["grad_out"] = _normal(seed, 47, (Q, H, d), dt)
        if c["packed"]:
            both = torch.empty(K, H + 2 * G, d, dtype=dt, device=DEV)
            s["grad_q"], s["grad_k"], s["grad_v"] = both[:, :H], both[:, H:H + G], both[:, H + G:]
        else:
            s["grad_q"], s["grad_k"], s["grad_v"] = (torch.empty_like(s[x]) for x in "qkv")
    return s


# ---- one pass ------------------------------------------------------------------------------------------------

_kept = {}


def _context():
    """The context that a program creates once."""
    if "ctx" not in _kept:
        from paper_2211_05239_amd import recd
        _kept["ctx"] = recd.Context(0)
    return _kept["ctx"]


def run(state):
    kind = state["case"]["kind"]
    if not own:
        return {"norm": _plain_norm, "loss": _plain_loss, "attention": _plain_attention}[kind](state)
    s, ctx, train = state, _context(), state["case"]["train"]
    if kind == "norm":
        if not train:
            ctx.layer_norm(s["x"], s["weight"], s["bias"], EPS, s["y"])
            return {"y": s["y"]}
        ctx.layer_norm(s["x"], s["weight"], s["bias"], EPS, s["y"], s["stats"])
        ctx.layer_norm_backward(s["x"], s["weight"], s["stats"], s["grad_y"], s["grad_x"], s["grad_weight"], s["grad_bias"])
        return {x: s[x] for x in ("y", "grad_x", "grad_weight", "grad_bias")}
    if kind == "loss":
        if not train:
            ctx.vocab_loss(s["x"], s["table"], s["targets"], s["scale"], s["loss"], s["lse"])
            return {"loss": s["loss"], "lse": s["lse"]}
        ctx.vocab_loss(s["x"], s["table"], s["targets"], s["scale"], s["loss"], s["lse"], s["mean_row"])
        ctx.vocab_loss_backward(s["x"], s["table"], s["targets"], s["scale"], s["lse"], s["mean_row"], s["grad_loss"],
                                s["grad_x"], s["grad_table"])
        return {x: s[x] for x in ("loss", "lse", "grad_x", "grad_table")}
    how = dict(scale=s["scale"], softcap=s["case"]["softcap"], slopes=s["slopes"], causal=s["case"]["causal"],
               prefix=s["prefix"])
    ctx.list_attention(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"], s["max_q"], s["max_k"], s["out"], s["lse"],
                       **how)
    if not train:
        return {"out": s["out"]}
    ctx.list_attention_backward(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"], s["max_q"], s["max_k"], s["out"],
                                s["lse"], s["grad_out"], s["grad_q"], s["grad_k"], s["grad_v"], **how)
    return {x: s[x] for x in ("out", "grad_q", "grad_k", "grad_v")}


# ---- the plain forms, in 32 bits -----------------------------------------------------------------------------

def _plain_norm(s):
    dt, x = s["x"].dtype, s["x"].float()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = (c.square().mean(1, keepdim=True) + EPS).rsqrt()
    h = c * rstd
    y = (h * s["weight"] + s["bias"]).to(dt)
    if not s["case"]["train"]:
        return {"y": y}
    g = s["grad_y"].float()
    gw = g * s["weight"]
    gx = rstd * (gw - gw.mean(1, keepdim=True) - h * (gw * h).mean(1, keepdim=True))
    return {"y": y, "grad_x": gx.to(dt), "grad_weight": (g * h).sum(0), "grad_bias": g.sum(0)}


def _plain_loss(s):
    dt, x, table, t = s["x"].dtype, s["x"].float(), s["table"].float(), s["targets"]
    z = torch.matmul(x, table.t()).mul_(s["scale"])
    has, at = t >= 0, t.clamp(min=0)
    picked = z.gather(1, at[:, None])[:, 0]
    top = z.amax(1)
    p = z.sub_(top[:, None]).exp_()
    total = p.sum(1)
    lse = top + total.log()
    loss = torch.where(has, lse - picked, 0.0)
    if not s["case"]["train"]:
        return {"loss": loss, "lse": lse}
    g = torch.where(has, s["grad_loss"] * s["scale"], 0.0)
    dz = p.mul_((g / total)[:, None])
    dz.scatter_add_(1, at[:, None], -g[:, None])
    return {"loss": loss, "lse": lse, "grad_x": torch.matmul(dz, table).to(dt), "grad_table": torch.matmul(dz.t(), x).to(dt)}


def _padded(x, offsets, most):
    """Rows [lists, most, heads, head_dim] in 32 bits, where each row stands, and which ones are rows of the list."""
    lens = offsets[1:] - offsets[:-1]
    at = torch.arange(most, device=DEV)
    there = at < lens[:, None]
    index = torch.where(there, offsets[:-1, None] + at, 0)
    rows = x[index].float() if x.shape[0] else x.new_zeros((*index.shape, *x.shape[1:]), dtype=torch.float32)
    return torch.where(there[..., None, None], rows, 0.0).transpose(1, 2), there


def _plain_attention(s):
    c, dt = s["case"], s["q"].dtype
    H, G = c["heads"], c["kv_heads"]
    q, q_there = _padded(s["q"], s["q_offsets"], s["max_q"])
    k, k_there = _padded(s["k"], s["k_offsets"], s["max_k"])
    v, _ = _padded(s["v"], s["k_offsets"], s["max_k"])
    k, v = k.repeat_interleave(H // G, 1), v.repeat_interleave(H // G, 1)
    nq, nk = s["q_offsets"].diff(), s["k_offsets"].diff()
    i, j = torch.arange(s["max_q"], device=DEV), torch.arange(s["max_k"], device=DEV)
    pos = (nk - nq)[:, None] + i                                           # a list's last query stands at its last key
    sees = q_there[:, :, None] & k_there[:, None, :]
    if c["causal"]:
        past = j <= pos[:, :, None]
        if s["prefix"] is not None:
            past = past | (j < s["prefix"][:, None, None])
        sees = sees & past
    z = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"])
    cap = c["softcap"]
    if cap:
        z = z.div_(cap).tanh_()
        slope = 1.0 - z * z if c["train"] else None                        # the cap's derivative
        z = z.mul_(cap)
    if s["slopes"] is not None:
        far = (pos[:, :, None] - j).abs().float()
        z = z.sub_(far[:, None] * s["slopes"][:, None, None])
    z = z.masked_fill_(~sees[:, None], -math.inf)
    top = z.amax(3, keepdim=True)
    p = z.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    p = p.div_(p.sum(3, keepdim=True).clamp(min=1e-30))                    # 0 where a row sees nothing
    out = torch.matmul(p, v)

    def rows(x, there):                                                    # back to the jagged rows
        return x.transpose(1, 2)[there].to(dt)

    if not c["train"]:
        return {"out": rows(out, q_there)}
    g, _ = _padded(s["grad_out"], s["q_offsets"], s["max_q"])
    L, _, mk, d = k.shape

    def shared(x):                                                         # the sum over the heads that share a key head
        return x.reshape(L, G, H // G, mk, d).sum(2)

    gv = shared(torch.matmul(p.transpose(2, 3), g))
    dz = torch.matmul(g, v.transpose(2, 3)).sub_((g * out).sum(3, keepdim=True)).mul_(p)
    del p, z
    dz = dz.mul_(s["scale"]) if not cap else dz.mul_(slope).mul_(s["scale"])
    return {"out": rows(out, q_there), "grad_q": rows(torch.matmul(dz, k), q_there),
            "grad_k": rows(shared(torch.matmul(dz.transpose(2, 3), q)), k_there), "grad_v": rows(gv, k_there)}


# ---- what a pass cannot do without ---------------------------------------------------------------------------

def work(case):
    c, e = case, SIZE[case["dtype"]]
    if c["kind"] == "norm":
        n, D = c["n"], c["D"]
        # the forward pass reads a row and writes one; the backward reads two, writes one and the summed gradients
        return {"bytes": n * D * e * (5 if c["train"] else 2) + D * 4 * (5 if c["train"] else 2), "flops": n * D * (20 if c["train"] else 8)}
    if c["kind"] == "loss":
        n, V, D = c["n"], c["rows"], c["D"]
        data = (n + V) * D * e
        return {"bytes": data * (2 if c["train"] else 1) + n * (8 + 4 + 4 + (4 if c["train"] else 0)),
                "flops": 2 * n * V * D * (3 if c["train"] else 1)}
    nq, nk = _lengths(c)
    H, G, d = c["heads"], c["kv_heads"], c["head_dim"]
    prefix = _prefixes(c, nk) if c["prefix"] else np.zeros_like(nk)
    pairs = 0
    for a, b, p in zip(nq.tolist(), nk.tolist(), prefix.tolist()):
        if not c["causal"]:
            pairs += a * b
        else:
            i = np.arange(a)
            pairs += int(np.clip(np.maximum(b - a + i + 1, p), 0, b).sum())
    Q, K = int(nq.sum()), int(nk.sum())
    once = (2 * Q * H + 2 * K * G) * d * e                                 # q, k, v read and out written
    lists = 16 * (c["lists"] + 1)
    # two products forward, four more backward; the backward pass reads grad_out and writes three gradients
    return {"bytes": lists + once + ((2 * Q * H + 2 * K * G) * d * e if c["train"] else 0),
            "flops": 2 * pairs * H * d * (6 if c["train"] else 2)}


# ---- the same in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    c, s = case, prepare(case, seed)
    f64 = torch.float64
    if c["kind"] == "norm":
        x, w, b = (s[n].to(f64).requires_grad_(c["train"]) for n in ("x", "weight", "bias"))
        y = torch.nn.functional.layer_norm(x, (c["D"],), w, b, EPS)
        if not c["train"]:
            return {"y": y}
        y.backward(s["grad_y"].to(f64))
        return {"y": y.detach(), "grad_x": x.grad, "grad_weight": w.grad, "grad_bias": b.grad}
    if c["kind"] == "loss":
        V = c["rows"]
        table = s["table"].to(f64).requires_grad_(c["train"])
        loss, lse, grad_x = [], [], []
        step = max(1, int(4e8) // V)                                       # 3 GB of logits at a time
        for i in range(0, c["n"], step):
            x = s["x"][i:i + step].to(f64).requires_grad_(c["train"])
            z = torch.nn.functional.linear(x, table) * s["scale"]
            one = torch.nn.functional.cross_entropy(z, s["targets"][i:i + step], ignore_index=-1, reduction="none")
            loss.append(one.detach())
            lse.append(torch.logsumexp(z.detach(), 1))
            if c["train"]:
                one.backward(s["grad_loss"][i:i + step].to(f64))
                grad_x.append(x.grad)
            del z, one
        got = {"loss": torch.cat(loss), "lse": torch.cat(lse)}
        return {**got, "grad_x": torch.cat(grad_x), "grad_table": table.grad} if c["train"] else got
    H, G, cap = c["heads"], c["kv_heads"], c["softcap"]
    # list by list: what the longest lists and the most lists take
    if c["lists"] > 10_000 or float(c["lists"]) * c["k_max"] * s["max_q"] * H > 4e9:
        return None
    q, k, v = (s[n].to(f64) for n in "qkv")
    out = torch.zeros(s["out"].shape, dtype=f64, device=DEV)
    grads = [torch.zeros(x.shape, dtype=f64, device=DEV) for x in (q, k, v)]
    go = s["grad_out"].to(f64) if c["train"] else None
    prefix = s["prefix"].tolist() if s["prefix"] is not None else [0] * c["lists"]
    qo, ko = s["q_offsets"].tolist(), s["k_offsets"].tolist()
    for a, b, e, f, pre in zip(qo, qo[1:], ko, ko[1:], prefix):
        nq, nk = b - a, f - e
        if nq == 0 or nk == 0:
            continue
        qs, ks, vs = q[a:b].transpose(0, 1), k[e:f].transpose(0, 1), v[e:f].transpose(0, 1)
        qs = qs.reshape(G, H // G * nq, -1)                                # a key head's queries together
        z = torch.bmm(qs, ks.transpose(1, 2).contiguous()).view(H, nq, nk) * s["scale"]
        if cap:
            t = torch.tanh(z / cap)
            z = cap * t
        pos = torch.arange(nk - nq, nk, device=DEV)[:, None]
        j = torch.arange(nk, device=DEV)
        if s["slopes"] is not None:
            z = z - s["slopes"].to(f64)[:, None, None] * (pos - j).abs().to(f64)
        if c["causal"]:
            z = torch.where((j <= pos) | (j < pre), z, -math.inf)
        p = torch.nan_to_num(torch.softmax(z, 2), nan=0.0)
        pg = p.reshape(G, H // G * nq, nk)
        o = torch.bmm(pg, vs.contiguous())
        out[a:b] = o.view(H, nq, -1).transpose(0, 1)
        if not c["train"]:
            continue
        gs = go[a:b].transpose(0, 1).reshape(G, H // G * nq, -1).contiguous()
        grads[2][e:f] = torch.bmm(pg.transpose(1, 2).contiguous(), gs).transpose(0, 1)
        dp = torch.bmm(gs, vs.transpose(1, 2).contiguous())
        dz = (pg * (dp - (pg * dp).sum(2, keepdim=True))).view(H, nq, nk)
        dz = (dz * (1 - t * t) if cap else dz) * s["scale"]
        dz = dz.reshape(G, H // G * nq, nk)
        grads[0][a:b] = torch.bmm(dz, ks.contiguous()).view(H, nq, -1).transpose(0, 1)
        grads[1][e:f] = torch.bmm(dz.transpose(1, 2).contiguous(), qs.contiguous()).transpose(0, 1)
    if not c["train"]:
        return {"out": out}
    return {"out": out, "grad_q": grads[0], "grad_k": grads[1], "grad_v": grads[2]}
