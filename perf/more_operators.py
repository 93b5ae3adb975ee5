"""Dense layers, dropout and answers on the rows of deduplicated lists, as cases to be measured.

What a next-id model does with its rows beside the norms, the attention and the loss:

  dropout  out = residual + x * mask / (1 - p), where the mask is made of a counter (row, column, call) and is never stored;
           its gradient makes the mask again
  dense    y = residual + dropout(act(x w^T + bias)); its gradients by x, w and bias, from sums x w^T + bias that the program
           kept (where a row of x is long) or that are made again (where it is not)
  answers  of every row scored against a whole table: the log probability of a given id, the entropy, and the k most likely
           ids with their log probabilities

The mask: eight elements of a row share the 128 bits that the counter generator Philox 4x32 with 10 rounds (Salmon et al., 2011)
makes of the key `seed` and the counter (column / 8, row, call), 16 bits each in their order; an element stays where its bits are
not below p * 2^16.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
CALL = 11          # the call's number within a training step


def _dropout(name, dtype, n, D, p, residual):
    return {"name": name, "kind": "dropout", "dtype": dtype, "n": n, "D": D, "p": p, "residual": residual}


def _dense(name, dtype, n, inner, outer, act, bias, p, residual, strided, train, kept=False):
    """train: no ReLU, whose slope jumps where 32 bits cannot tell on which side of 0 a sum lies."""
    return {"name": name, "kind": "dense", "dtype": dtype, "n": n, "in": inner, "out": outer, "act": act, "bias": bias, "p": p,
            "residual": residual, "strided": strided, "train": train, "kept": kept}


def _answers(name, dtype, n, rows, D, k):
    return {"name": name, "kind": "answers", "dtype": dtype, "n": n, "rows": rows, "D": D, "k": k}


def listed():
    return [
        # a small batch's rows, training: launches count
        _dropout("dropout_small_f16", "f16", 301, 64, 0.1, True),
        # the unique ids of a training batch (benchmark configuration 2), behind a layer's output
        _dropout("dropout_train_bf16", "bf16", 300_007, 128, 0.1, True),
        # the embeddings of wide fp32 rows
        _dropout("dropout_wide_f32", "f32", 50_021, 516, 0.5, False),
        # one new position of each of 37 histories through the first layer of a feed-forward block: serving
        _dense("dense_tokens_f16", "f16", 37, 128, 512, "gelu", True, 0.0, False, False, False),
        # one request's pooled features (64 of 128, configuration 5) into the first layer of a model above them: serving
        _dense("dense_single_bf16", "bf16", 1, 8192, 1024, "relu", True, 0.0, False, False, False),
        # training of a feed-forward block on the unique ids of a batch: its first layer
        _dense("dense_up_bf16", "bf16", 300_007, 128, 512, "gelu", True, 0.1, False, False, True),
        # and its second one, back onto the rows
        _dense("dense_down_bf16", "bf16", 300_007, 512, 128, "none", True, 0.1, True, False, True),
        # the largest: training of the layer above the pooled features of a batch (configuration 5: 16 384 rows)
        _dense("dense_pooled_bf16", "bf16", 16_384, 8192, 1024, "silu", True, 0.0, False, False, True, True),
        # fp32 training, odd widths, rows inside of wider ones
        _dense("dense_ragged_f32", "f32", 5021, 516, 260, "silu", True, 0.0, True, True, True),
        # a request's last positions and their ten best ids out of 100 K
        _answers("answers_request_f32", "f32", 37, 100_000, 64, 10),
        # evaluation against an odd table in 16 bits: is the best id the right one
        _answers("answers_ragged_f16", "f16", 2500, 300_007, 96, 1),
        # evaluation against a table of a million rows of 128 (configurations 2 to 5), with alternatives
        _answers("answers_large_bf16", "bf16", 4096, 1_000_000, 128, 8),
    ]


def draw(rng):
    """One more case of the same ranges: no larger than the largest listed one of its kind."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["dropout", "dense", "dense", "answers"])
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    per = 4 if dtype == "f32" else 8   # values of a 16-byte piece
    if kind == "dropout":
        D = per * log(1, 256)
        c = _dropout("", dtype, min(log(1, 400_000), 38_000_000 // D), D, rng.choice([0.05, 0.1, 0.2, 0.5]), rng.random() < 0.5)
    elif kind == "dense":
        inner, outer = per * log(2, 8192 // per), per * log(2, 4096 // per)
        most = 1.3e11 if dtype != "f32" else 1.3e10
        n = max(1, min(log(1, 400_000), int(most / (inner * outer)), int(1.5e8 / (inner + outer))))
        train = rng.random() < 0.6
        act = rng.choice(["none", "gelu", "gelu", "silu"] if train else ["none", "relu", "gelu", "silu"])
        c = _dense("", dtype, n, inner, outer, act, rng.random() < 0.8, rng.choice([0.0, 0.1, 0.5]) if train else 0.0,
                   rng.random() < 0.4, rng.random() < 0.3, train, train and act != "none" and inner >= 1024)
    else:
        D = min(256, per * log(2, 64))
        rows = log(1000, 1_000_000)
        most = 4e9 / rows if dtype != "f32" else 4e8 / rows
        c = _answers("", dtype, max(1, min(log(1, 8192), int(most * min(1, 128 / D)))), rows, D, rng.choice([1, 4, 8, 10, 32, 50]))
    del c["name"]
    return c


# ---- inputs --------------------------------------------------------------------------------------------------

def _gen(seed, tag):
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * int(seed) + tag)
    return g


def _normal(seed, tag, shape, dtype, std=1.0, mean=0.0):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(mean, std, generator=_gen(seed, tag))


def _rows(c, x):
    """x, in the middle of wider rows where the case has its rows strided."""
    if not c["strided"]:
        return x
    wide = torch.empty(x.shape[0], x.shape[1] + 48, dtype=x.dtype, device=DEV)
    wide[:, 32:-16] = x
    return wide[:, 32:-16]


def prepare(case, seed):
    c, dt = case, DTYPE[case["dtype"]]
    s = {"case": c, "seed": 7_919 * int(seed) + (int(seed) << 34) + 1}
    if c["kind"] == "dropout":
        shape = c["n"], c["D"]
        s["x"], s["grad_out"] = _normal(seed, 3, shape, dt, 1.5, 0.3), _normal(seed, 5, shape, dt)
        s["residual"] = _normal(seed, 7, shape, dt) if c["residual"] else None
        s["out"], s["grad_x"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        return s
    if c["kind"] == "dense":
        n, inner, outer = c["n"], c["in"], c["out"]
        s["x"] = _rows(c, _normal(seed, 11, (n, inner), dt))
        s["w"] = _normal(seed, 13, (outer, inner), dt, 1.0 / math.sqrt(inner))
        s["bias"] = _normal(seed, 17, (outer,), torch.float32, 0.2) if c["bias"] else None
        s["residual"] = _rows(c, _normal(seed, 19, (n, outer), dt)) if c["residual"] else None
        s["y"] = _rows(c, torch.zeros(n, outer, dtype=dt, device=DEV))
        if c["train"]:
            s["grad_y"] = _rows(c, _normal(seed, 23, (n, outer), dt))
            s["grad_x"] = _rows(c, torch.zeros(n, inner, dtype=dt, device=DEV))
            s["grad_w"] = torch.empty_like(s["w"])
            s["grad_bias"] = torch.empty_like(s["bias"]) if c["bias"] else None
        s["sums"] = torch.empty(n, outer, device=DEV) if c["kept"] else None
        return s
    n, V, D, k = c["n"], c["rows"], c["D"], c["k"]
    # rows behind a layer norm, a table whose logits spread by about two
    s["x"], s["table"], s["scale"] = _normal(seed, 29, (n, D), dt), _normal(seed, 31, (V, D), dt, 2.0 / math.sqrt(D)), 1.0
    u = torch.rand(n, generator=_gen(seed, 37), device=DEV, dtype=torch.float64)
    s["given"] = ((V ** u - 1).to(torch.int64).clamp_(0, V - 1) * 7919) % V        # about 1/k, as ids are
    s["logp"], s["entropy"], s["lse"] = (torch.empty(n, device=DEV) for _ in range(3))
    s["top_ids"], s["top_logp"] = torch.empty(n, k, dtype=torch.int64, device=DEV), torch.empty(n, k, device=DEV)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------

_kept = {}


def _context():
    """The context that a program creates once."""
    if "ctx" not in _kept:
        from paper_2211_05239_amd import recd
        _kept["ctx"] = recd.Context(0)
        _kept["Dropout"] = recd.Dropout
    return _kept["ctx"]


def run(state):
    kind = state["case"]["kind"]
    if not own:
        return {"dropout": _plain_dropout, "dense": _plain_dense, "answers": _plain_answers}[kind](state)
    s, c, ctx = state, state["case"], _context()
    if kind == "dropout":
        drop = _kept["Dropout"](c["p"], s["seed"], CALL)
        ctx.dropout(s["x"], drop, s["out"], residual=s["residual"])
        ctx.dropout_backward(s["grad_out"], drop, s["grad_x"])
        return {"out": s["out"], "grad_x": s["grad_x"]}
    if kind == "dense":
        how = dict(act=c["act"], dropout=_kept["Dropout"](c["p"], s["seed"], CALL) if c["p"] else None)
        ctx.dense(s["x"], s["w"], s["bias"], s["y"], residual=s["residual"], sums=s["sums"], **how)
        if not c["train"]:
            return {"y": s["y"]}
        ctx.dense_backward(s["x"], s["w"], s["bias"], s["grad_y"], s["grad_x"], s["grad_w"], s["grad_bias"], sums=s["sums"],
                           **how)
        return {x: s[x] for x in ("y", "grad_x", "grad_w", "grad_bias")}
    ctx.vocab_answers(s["x"], s["table"], s["scale"], s["given"], s["logp"], s["entropy"], s["lse"], s["top_ids"], s["top_logp"])
    return {x: s[x] for x in ("logp", "entropy", "lse", "top_ids", "top_logp")}


# ---- the plain forms, in 32 bits -----------------------------------------------------------------------------

def _cut(p):
    """Bits below this drop an element, and what scales the others."""
    t = int(math.floor(p * 65536 + 0.5))
    return t, 65536.0 / (65536 - t)


def _keep(n, D, p, seed):
    """[n, D]: whether an element stays."""
    low = 0xFFFFFFFF
    col = torch.arange((D + 7) // 8, device=DEV)
    row = torch.arange(n, device=DEV)[:, None]
    a, b, c, d = (x.expand(n, len(col)) for x in (col, row, torch.full_like(row, CALL), torch.zeros_like(row)))
    k0, k1 = seed & low, seed >> 32 & low
    for _ in range(10):
        u, v = a * 0xD2511F53, c * 0xCD9E8D57                              # the products' low 64 bits
        a, b, c, d = (v >> 32 & low) ^ b ^ k0, v & low, (u >> 32 & low) ^ d ^ k1, u & low
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    words = torch.stack([a, b, c, d], 2)
    bits = torch.stack([words & 0xFFFF, words >> 16], 3).reshape(n, -1)[:, :D]
    return bits >= _cut(p)[0]


def _plain_dropout(s):
    c, dt = s["case"], s["x"].dtype
    keep, by = _keep(c["n"], c["D"], c["p"], s["seed"]), _cut(c["p"])[1]
    out = torch.where(keep, s["x"].float() * by, 0.0)
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return {"out": out.to(dt), "grad_x": torch.where(keep, s["grad_out"].float() * by, 0.0).to(dt)}


def _act(act, z, slope):
    """The activation of z, and its derivative where that is asked for."""
    if act == "none":
        return z, torch.ones_like(z) if slope else None
    if act == "relu":
        return z.clamp(min=0.0), (z > 0).float() if slope else None
    if act == "silu":
        g = 1.0 / (1.0 + torch.exp(-z))
        return z * g, g * (1.0 + z * (1.0 - g)) if slope else None
    g = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z * g, g + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi)) if slope else None


def _plain_dense(s):
    c, dt = s["case"], s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    z = torch.matmul(x, w.t())
    if s["bias"] is not None:
        z = z + s["bias"]
    h, slope = _act(c["act"], z, c["train"])
    keep, by = (_keep(c["n"], c["out"], c["p"], s["seed"]), _cut(c["p"])[1]) if c["p"] else (None, 1.0)
    if keep is not None:
        h = torch.where(keep, h * by, 0.0)
    if s["residual"] is not None:
        h = h + s["residual"].float()
    if not c["train"]:
        return {"y": h.to(dt)}
    g = s["grad_y"].float() * slope
    if keep is not None:
        g = torch.where(keep, g * by, 0.0)
    grad_bias = g.sum(0) if s["bias"] is not None else None
    return {"y": h.to(dt), "grad_x": torch.matmul(g, w).to(dt), "grad_w": torch.matmul(g.t(), x).to(dt), "grad_bias": grad_bias}


def _plain_answers(s):
    x, table, k = s["x"], s["table"], s["case"]["k"]
    z = torch.matmul(x.float(), table.float().t()).mul_(s["scale"])
    logp = z.gather(1, s["given"][:, None])[:, 0]
    # some more than k by 32 bits, put in order by 64: neighbours in rank are often nearer than 32 bits tell apart
    ids = z.topk(min(k + 16, z.shape[1]), 1).indices.sort(1).values
    top = z.amax(1, keepdim=True)
    z = z.sub_(top)
    p = z.exp()
    total = p.sum(1)
    entropy = total.log() - p.mul_(z).sum(1) / total
    lse = top[:, 0] + total.log()
    best = (table[ids].double() * x.double()[:, None]).sum(2) * s["scale"]
    best, at = best.sort(stable=True, dim=1, descending=True)
    return {"logp": logp - lse, "entropy": entropy, "lse": lse, "top_ids": ids.gather(1, at)[:, :k].contiguous(),
            "top_logp": (best[:, :k] - lse.double()[:, None]).float()}


# ---- what a pass cannot do without ---------------------------------------------------------------------------

def work(case):
    c, e = case, SIZE[case["dtype"]]
    if c["kind"] == "dropout":
        # forward reads a row (and the residual's) and writes one, backward reads one and writes one
        return {"bytes": c["n"] * c["D"] * e * (5 if c["residual"] else 4), "flops": c["n"] * c["D"] * 4}
    if c["kind"] == "dense":
        n, inner, outer, train = c["n"], c["in"], c["out"], c["train"]
        once = n * inner + inner * outer + n * outer * (2 if c["residual"] else 1)
        back = n * outer + n * inner + inner * outer if train else 0
        return {"bytes": (once + back) * e + (outer * 4 * (2 if train else 1) if c["bias"] else 0),
                "flops": 2 * n * inner * outer * (3 if train else 1)}
    n, V, D, k = c["n"], c["rows"], c["D"], c["k"]
    return {"bytes": (n + V) * D * e + n * (8 + 4 * 3 + k * 12), "flops": 2 * n * V * D}


# ---- the same in 64 bits -------------------------------------------------------------------------------------

def _exact_keep(n, D, p, seed):
    """The mask again, of 64-bit words on the host."""
    w = np.uint64
    low = w(0xFFFFFFFF)
    pieces = -(-D // 8)
    at = np.arange(n * pieces, dtype=w)
    ctr = [at % w(pieces), at // w(pieces), np.full(n * pieces, CALL, dtype=w), np.zeros(n * pieces, dtype=w)]
    key = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    for _ in range(10):
        first, second = ctr[0] * w(0xD2511F53), ctr[2] * w(0xCD9E8D57)
        ctr = [(second >> w(32)) ^ ctr[1] ^ w(key[0]), second & low, (first >> w(32)) ^ ctr[3] ^ w(key[1]), first & low]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    words = np.stack(ctr, 1).astype(np.uint32)
    bits = words.view(np.uint16).reshape(n, pieces * 8)[:, :D]              # little endian: the low half first
    return torch.from_numpy(bits >= round(p * 65536)).to(DEV)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    f64 = torch.float64
    if c["kind"] == "dropout":
        keep = _exact_keep(c["n"], c["D"], c["p"], s["seed"]).to(f64)
        keep = keep / (1.0 - round(c["p"] * 65536) / 65536.0)
        out = s["x"].to(f64) * keep
        return {"out": out + s["residual"].to(f64) if c["residual"] else out, "grad_x": s["grad_out"].to(f64) * keep}
    if c["kind"] == "dense":
        f = torch.nn.functional
        x, w = (s[n].to(f64).requires_grad_(c["train"]) for n in ("x", "w"))
        b = s["bias"].to(f64).requires_grad_(c["train"]) if c["bias"] else None
        y = {"none": lambda z: z, "relu": f.relu, "gelu": f.gelu, "silu": f.silu}[c["act"]](f.linear(x, w, b))
        if c["p"]:
            y = y * _exact_keep(c["n"], c["out"], c["p"], s["seed"]).to(f64) / (1.0 - round(c["p"] * 65536) / 65536.0)
        if c["residual"]:
            y = y + s["residual"].to(f64)
        if not c["train"]:
            return {"y": y}
        y.backward(s["grad_y"].to(f64))
        return {"y": y.detach(), "grad_x": x.grad, "grad_w": w.grad, "grad_bias": b.grad if c["bias"] else None}
    V, k = c["rows"], c["k"]
    table = s["table"].to(f64)
    got = {"logp": [], "entropy": [], "lse": [], "top_ids": [], "top_logp": []}
    step = max(1, int(4e8) // V)                                           # 3 GB of logits at a time
    for i in range(0, c["n"], step):
        logs = torch.log_softmax(torch.nn.functional.linear(s["x"][i:i + step].to(f64), table) * s["scale"], 1)
        got["logp"].append(logs.gather(1, s["given"][i:i + step, None])[:, 0])
        got["entropy"].append(torch.special.entr(logs.exp()).sum(1))
        # any logit is its log probability and the sum's logarithm
        first = (s["x"][i:i + step].to(f64) * table[0]).sum(1) * s["scale"]
        got["lse"].append(first - logs[:, 0])
        best = logs.topk(k, 1)
        got["top_ids"].append(best.indices)
        got["top_logp"].append(best.values)
    return {n: torch.cat(v) for n, v in got.items()}
