"""Plain 64-bit forms of the operators on rows of lists, with bounds of what fp32 sums and one rounding may do.

A bound is made from the reference alone: u is the unit roundoff of the outputs' type (also what the probabilities
are rounded by where they enter a product), E that of fp32.  Errors of first order are added up; 4 * E * (terms)
stands for a sum of that many terms in any order."""
import math

import torch

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 1e-37, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-37}   # what underflows
E = 2.0 ** -24


def within(got, ref, bound, what=""):
    assert got.shape == ref.shape, what
    g = got.double().cpu()
    err = (g - ref).abs()
    bad = ~(err <= bound + TINY[got.dtype] + U[got.dtype] * ref.abs() * 1.01)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst {float((err / (bound + 1e-300)).max()):.3g} of it"


def same_bits(a, b):
    whole = {4: torch.int32, 2: torch.int16}[a.element_size()]
    return torch.equal(a.contiguous().view(whole), b.contiguous().view(whole))


def rand(shape, dt, seed, std=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g, dtype=torch.float64) * std + mean).to(DT[dt])


# ---- layer norm -------------------------------------------------------------------------------------------------

def norm_ref(x, w, b, eps, g=None):
    """{name: (value, bound)}"""
    x = x.double()
    D = x.shape[1]
    w = torch.ones(D, dtype=torch.float64) if w is None else w.double()
    b = torch.zeros(D, dtype=torch.float64) if b is None else b.double()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = 1.0 / (c.square().mean(1, keepdim=True) + eps).sqrt()
    h = c * rstd
    n = 4 * E * (D + 8)
    # the mean is off by n/4 * mean|x|, every difference by that and a rounding, rstd by that part of the squares
    dc = n * x.abs().mean(1, keepdim=True) + 2 * E * x.abs()
    dh = dc * rstd + h.abs() * (n + (dc * c.abs()).mean(1, keepdim=True) * rstd * rstd * 2)
    out = {"y": (h * w + b, dh * w.abs() + 4 * E * (h * w).abs() + 4 * E * b.abs())}
    if g is None:
        return out
    g = g.double()
    u = g * w
    m1, m2 = u.mean(1, keepdim=True), (u * h).mean(1, keepdim=True)
    gx = rstd * (u - m1 - h * m2)
    dm1 = n * u.abs().mean(1, keepdim=True)
    dm2 = n * (u * h).abs().mean(1, keepdim=True) + (u.abs() * dh).mean(1, keepdim=True)
    rel = (dc * c.abs()).mean(1, keepdim=True) * rstd * rstd * 2 + n
    out["grad_x"] = (gx, rstd * (dm1 + dh * m2.abs() + h.abs() * dm2 + 8 * E * (u.abs() + m1.abs() + (h * m2).abs())) + rel * gx.abs())
    N = x.shape[0]
    out["grad_weight"] = ((g * h).sum(0), (g.abs() * dh).sum(0) + 4 * E * (N + 4) * (g * h).abs().sum(0))
    out["grad_bias"] = (g.sum(0), 4 * E * (N + 4) * g.abs().sum(0))
    return out


# ---- softmax cross entropy against a table ----------------------------------------------------------------------

def loss_ref(x, table, targets, scale, grad_loss=None):
    dt, D = x.dtype, x.shape[1]
    u = 0.0 if dt == torch.float32 else U[dt]
    x, table = x.double(), table.double()
    z = scale * (x @ table.t())
    size = abs(scale) * (x.abs() @ table.abs().t())
    lse = torch.logsumexp(z, 1)
    p = (z - lse[:, None]).exp()
    # a logit is off by the sum's error and by the steps of the exponent's argument
    dz = 4 * E * (D + 8) * size + 8 * E * (z.abs() + lse.abs()[:, None])
    dlse = (p * dz).sum(1) + 4 * E * (z.shape[1] + 8) + 4 * E * lse.abs()
    has = (targets >= 0) & (targets < table.shape[0])
    at = targets.clamp(0, table.shape[0] - 1)
    picked, dpicked = z.gather(1, at[:, None])[:, 0], dz.gather(1, at[:, None])[:, 0]
    out = {"lse": (lse, dlse), "loss": (torch.where(has, lse - picked, 0.0), torch.where(has, dlse + dpicked, 0.0))}
    if grad_loss is None:
        return out
    g = torch.where(has, grad_loss.double(), 0.0)
    dp = p * (dz + dlse[:, None] + 8 * E)                     # of a probability
    mean = p @ table
    dmean = (p * u + dp) @ table.abs() + 4 * E * (table.shape[0] + 8) * (p @ table.abs())
    gx = scale * g[:, None] * (mean - table[at])
    out["grad_x"] = (gx, abs(scale) * g.abs()[:, None] * (dmean + 4 * E * (mean.abs() + table[at].abs())))
    one = torch.zeros_like(p)
    one[has.nonzero()[:, 0], at[has]] = 1.0
    w = g[:, None] * (p - one)
    dw = g.abs()[:, None] * dp + u * w.abs() + 4 * E * (g[:, None] * (p + one)).abs()
    # fp16 products are held to 2^-38 of the largest weight (a power of two below 2^14 above it, and 2^-24 steps)
    dw = dw + (g.abs().max() * 2.0 ** -36 if dt == torch.float16 else 0.0)
    out["grad_table"] = (scale * (w.t() @ x), abs(scale) * (dw.t() @ x.abs() + 4 * E * (x.shape[0] + 8) * (w.abs().t() @ x.abs())))
    return out


# ---- attention inside lists -------------------------------------------------------------------------------------

def attention_ref(q, k, v, q_offsets, k_offsets, scale, softcap=0.0, slopes=None, causal=False, prefix=None, g=None):
    """q [Q, H, d], k and v [K, G, d] on the CPU; lists one by one, heads one by one."""
    dt, (Q, H, d), G = q.dtype, q.shape, k.shape[1]
    u = 0.0 if dt == torch.float32 else U[dt]
    q, k, v = q.double(), k.double(), v.double()
    z0 = lambda *s: torch.zeros(*s, dtype=torch.float64)  # noqa: E731
    out, dout, lse, dlse = z0(Q, H, d), z0(Q, H, d), torch.full((Q, H), -math.inf, dtype=torch.float64), z0(Q, H)
    grads = [z0(Q, H, d), z0(Q, H, d), z0(*k.shape), z0(*k.shape), z0(*v.shape), z0(*v.shape)]
    g = g.double() if g is not None else None
    qo, ko = q_offsets.tolist(), k_offsets.tolist()
    for l, (a, b, e, f) in enumerate(zip(qo, qo[1:], ko, ko[1:])):
        nq, nk = b - a, f - e
        if not nq or not nk:
            continue
        pos = torch.arange(nk - nq, nk)[:, None]
        j = torch.arange(nk)
        sees = torch.ones(nq, nk, dtype=torch.bool)
        if causal:
            sees = (j <= pos) | (j < (int(prefix[l]) if prefix is not None else 0))
        for h in range(H):
            qs, ks, vs = q[a:b, h], k[e:f, h // (H // G)], v[e:f, h // (H // G)]
            raw = scale * (qs @ ks.t())
            dz = 4 * E * (d + 8) * abs(scale) * (qs.abs() @ ks.abs().t()) + 8 * E * raw.abs()
            t = torch.zeros_like(raw)
            z = raw
            if softcap:
                t = torch.tanh(raw / softcap)
                z = softcap * t
                dz = dz + 8 * E * softcap
            if slopes is not None:
                far = float(slopes[h]) * (pos - j).abs()
                z = z - far
                dz = dz + 8 * E * (far.abs() + z.abs())
            z = z.masked_fill(~sees, -math.inf)
            some = sees.any(1)
            lse_h = torch.logsumexp(z, 1)
            p = torch.where(sees, (z - torch.where(some, lse_h, 0.0)[:, None]).exp(), 0.0)
            dl = (p * dz).sum(1) + 4 * E * (nk + 8) + 8 * E * torch.where(some, lse_h.abs(), 0.0)
            dp_rel = dz + dl[:, None] + 8 * E                       # relative, of a probability
            dp = p * dp_rel
            o = p @ vs
            out[a:b, h], lse[a:b, h], dlse[a:b, h] = o, lse_h, dl
            do = (p * u + dp) @ vs.abs() + 4 * E * (nk + 8) * (p @ vs.abs())
            dout[a:b, h] = do
            if g is None:
                continue
            gs = g[a:b, h]
            x = gs @ vs.t()
            dx = 4 * E * (d + 8) * (gs.abs() @ vs.abs().t())
            delta = (p * x).sum(1, keepdim=True)
            # delta comes from the rounded outputs
            ddelta = (gs.abs() * (do + u * o.abs())).sum(1, keepdim=True) + 4 * E * (d + 8) * (gs * o).abs().sum(1, keepdim=True)
            slope = 1 - t * t
            ds = scale * p * (x - delta) * slope
            dds = abs(scale) * slope * (dp * (x - delta).abs() + p * (dx + ddelta + 4 * E * (x.abs() + delta.abs()))) + u * ds.abs()
            if softcap:
                dds = dds + abs(scale) * p * (x - delta).abs() * 2 * t.abs() * (16 * E + dz / softcap)
            if dt == torch.float16:
                # ds is held to 2^-24 of 2^15 / bound, in powers of two
                dds = dds + abs(scale) * 2.0 ** -36 * 2 * d * float(g.abs().max()) * float(v.abs().max())
            grads[0][a:b, h], grads[1][a:b, h] = ds @ ks, dds @ ks.abs() + 4 * E * (nk + 8) * (ds.abs() @ ks.abs())
            grads[2][e:f, h // (H // G)] += ds.t() @ qs
            grads[3][e:f, h // (H // G)] += dds.t() @ qs.abs() + 4 * E * (nq * H + 8) * (ds.abs().t() @ qs.abs())
            grads[4][e:f, h // (H // G)] += p.t() @ gs
            pu = p * u + dp + (2.0 ** -39 if dt == torch.float16 else 0.0)
            grads[5][e:f, h // (H // G)] += pu.t() @ gs.abs() + 4 * E * (nq * H + 8) * (p.t() @ gs.abs())
    got = {"out": (out, dout), "lse": (lse, dlse)}
    if g is not None:
        got.update(grad_q=(grads[0], grads[1]), grad_k=(grads[2], grads[3]), grad_v=(grads[4], grads[5]))
    return got
