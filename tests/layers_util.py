"""Plain 64-bit forms of dense layers, dropout and answers, with bounds of what 32-bit sums and one rounding may do (u, E and the
rule for sums as in dense_util)."""
import math

import numpy as np
import torch

from tests.dense_util import E, U

LOW = 0xFFFFFFFF
# The vector units' exponential and reciprocal give 0 where the result is below the smallest normal number: a sigmoid or a tail of the
# normal distribution is off by up to that there (z < -87.3 and z < -12.9), and z times it by |z| times as much.
FLUSH = 2.0 ** -126 * 1.01


def philox(ctr, key):
    """Philox 4x32, 10 rounds, of counters [..., 4] and a key of two words, in Python's integers' arithmetic on uint64."""
    c = [np.asarray(ctr[..., i], dtype=np.uint64) for i in range(4)]
    k = [int(key[0]), int(key[1])]
    for _ in range(10):
        u, v = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(v >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), v & np.uint64(LOW), (u >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]),
             u & np.uint64(LOW)]
        k = [(k[0] + 0x9E3779B9) & LOW, (k[1] + 0xBB67AE85) & LOW]
    return np.stack(c, -1)


def cut(p):
    return math.floor(p * 65536 + 0.5)


def keep(n, D, p, seed, call, row0=0):
    """[n, D]: whether an element stays."""
    pieces = -(-D // 8)
    rows = (np.arange(n, dtype=np.uint64) + np.uint64(row0))[:, None]
    cols = np.arange(pieces, dtype=np.uint64)[None]
    call &= (1 << 64) - 1
    one = np.ones((n, pieces), dtype=np.uint64)
    ctr = np.stack([(cols + ((rows >> np.uint64(32)) << np.uint64(16))) & np.uint64(LOW), (rows & np.uint64(LOW)) * one,
                    one * np.uint64(call & LOW), one * np.uint64(call >> 32)], -1)
    w = philox(ctr, (seed & LOW, seed >> 32 & LOW)).astype(np.uint32)
    halves = np.stack([w & 0xFFFF, w >> 16], -1).reshape(n, pieces * 8)[:, :D]
    return torch.from_numpy(halves >= cut(p))


def dropout_ref(x, p, seed, call, residual=None, row0=0):
    """(value, bound)"""
    by = 65536.0 / (65536 - cut(p))
    h = torch.where(keep(*x.shape, p, seed, call, row0), x.double() * by, 0.0)
    r = residual.double() if residual is not None else torch.zeros_like(h)
    return h + r, 4 * E * (h.abs() + r.abs())


def _act(act, z):
    """act(z), its slope, what 32 bits may be off by in either, and the curvature's bound."""
    if act == "none":
        return z, torch.ones_like(z), 0 * z, 0 * z, 0.0
    if act == "relu":
        return z.clamp(min=0), (z > 0).double(), 0 * z, 0 * z, 0.0
    if act == "silu":
        # the exponential: its argument's rounding and its own, the reciprocal's
        s = torch.sigmoid(z)
        rel = 8 * E + 2 * E * z.abs()
        return z * s, s * (1 + z * (1 - s)), (z * s).abs() * (rel + E) + z.abs() * FLUSH, s * (1 + z.abs()) * 2 * rel, 0.5
    # P(-|z|): 2.8 E of the polynomial, its steps' roundings (their terms add up to 1.8 times its value at most), the reciprocal's and
    # the exponential's, whose argument grows with z^2
    P = 0.5 * torch.erfc(-z / math.sqrt(2))
    tail = 0.5 * torch.erfc(z.abs() / math.sqrt(2))
    phi = torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    rel = 32 * E + 2 * E * z * z
    return (z * P, P + z * phi, z.abs() * tail * rel + 4 * E * (z * P).abs() + z.abs() * FLUSH,
            tail * rel + (z * phi).abs() * (4 * E + 2 * E * z * z) + 4 * E, 0.8)


def dense_ref(x, w, bias=None, act="none", p=0.0, seed=0, call=0, residual=None, g=None):
    """{name: (value, bound)} on the CPU."""
    dt, (n, K), N = x.dtype, x.shape, w.shape[0]
    u = 0.0 if dt == torch.float32 else U[dt]
    x, w = x.double(), w.double()
    b = torch.zeros(N, dtype=torch.float64) if bias is None else bias.double()
    z = x @ w.t() + b
    dz = 4 * E * (K + 8) * (x.abs() @ w.abs().t()) + 4 * E * (b.abs() + z.abs())
    h, slope, dh, dslope, curve = _act(act, z)
    dh = dh + 1.2 * dz
    by = 65536.0 / (65536 - cut(p))
    mask = keep(n, N, p, seed, call).double() * by if p else torch.ones(n, N, dtype=torch.float64)
    r = residual.double() if residual is not None else torch.zeros_like(z)
    out = {"y": (mask * h + r, mask * dh + 4 * E * ((mask * h).abs() + r.abs())), "sums": (z, dz)}
    if g is None:
        return out
    g = g.double()
    gz = g * mask * slope
    dgz = (g * mask).abs() * (dslope + curve * dz) + 4 * E * gz.abs()
    if act == "relu":
        dgz = dgz + (g * mask).abs() * (z.abs() <= dz)             # either side of the jump
    out["grad_bias"] = (gz.sum(0), dgz.sum(0) + 4 * E * (n + 8) * gz.abs().sum(0))
    into = dgz
    if act != "none" or p:
        into = into + u * gz.abs() + (2.0 ** -25 if dt == torch.float16 else 0.0)
    out["grad_x"] = (gz @ w, into @ w.abs() + 4 * E * (N + 8) * (gz.abs() @ w.abs()))
    out["grad_w"] = (gz.t() @ x, into.t() @ x.abs() + 4 * E * (n + 8) * (gz.abs().t() @ x.abs()))
    return out


def logits(x, table, scale):
    """[n, V] in 64 bits, every logit by sums of the same order, so that equal rows of the table have equal ones."""
    x, table = x.double(), table.double()
    return torch.stack([(table * row).sum(1) for row in x]) * scale if len(x) else x.new_zeros(0, len(table))


def answers_ref(x, table, scale, given, k, z=None):
    """{name: (value, bound)}, and the ids."""
    D, V = x.shape[1], len(table)
    z = logits(x, table, scale) if z is None else z
    size = abs(scale) * (x.double().abs() @ table.double().abs().t())
    lse = torch.logsumexp(z, 1)
    p = (z - lse[:, None]).exp()
    dz = 4 * E * (D + 8) * size + 8 * E * (z.abs() + lse.abs()[:, None])
    dlse = (p * dz).sum(1) + 4 * E * (V + 8) + 4 * E * lse.abs()
    has = (given >= 0) & (given < V)
    picked = z.gather(1, given.clamp(0, V - 1)[:, None])[:, 0]
    H = torch.special.entr(p).sum(1)
    # the slope of H by a logit is -p (log p + H); both of its terms are positive, of sums of V terms
    dH = ((p * (z - lse[:, None] + H[:, None]).abs()) * dz).sum(1) + 4 * E * (V + 8) * (1 + H)
    out = {"lse": (lse, dlse), "logp": (torch.where(has, picked - lse, 0.0), torch.where(has, dlse + E * picked.abs(), 0.0)),
           "entropy": (H, dH)}
    best, ids = z.sort(dim=1, descending=True, stable=True)
    out["top_logp"] = (best[:, :k] - lse[:, None], dlse[:, None] + E * best[:, :k].abs())
    return out, ids[:, :k]
