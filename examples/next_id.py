"""Trains a next-id model on session-structured lists, with everything computed once per unique list.

A batch's lists of one feature are deduplicated; the rows of the unique lists are looked up, normalised, attend to the
rows before them in their list, and are scored against the whole table: row i of a list is to predict id i + 1.  A
unique list's loss counts as often as the batch holds the list, so loss and gradients are those of the whole batch.

    python examples/next_id.py [--steps 50] [--dtype f32|f16|bf16]
"""
import argparse
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2211_05239_amd import recd, synth  # noqa: E402

EPS = 1e-5
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


class Lists:
    """The unique lists of a batch: ids, offsets, how many of the batch's rows hold each list, next ids."""

    def __init__(self, ctx, values, offsets):
        B, N = offsets.numel() - 1, values.numel()
        self.ids = torch.empty(max(N, 1), dtype=torch.int64, device="cuda")
        self.offsets = torch.empty(B + 1, dtype=torch.int64, device="cuda")
        self.inverse = torch.empty(B, dtype=torch.int32, device="cuda")
        self.feat_uoff = torch.empty(2, dtype=torch.int64, device="cuda")
        self.U, self.M = ctx.build_ikjt(1, B, values, offsets, self.ids, self.offsets, self.inverse, self.feat_uoff,
                                        want_counts=True)
        self.ids, self.offsets = self.ids[:self.M], self.offsets[:self.U + 1]
        lens = self.offsets.diff()
        self.longest = int(lens.max()) if self.U else 0
        self.targets = torch.cat([self.ids[1:], self.ids.new_full((1,), -1)])[:self.M]
        self.targets[self.offsets[1:][lens > 0] - 1] = -1                  # the last row of a list has no next id
        counts = torch.bincount(self.inverse.long(), minlength=self.U).float()
        self.weight = torch.repeat_interleave(counts, lens, output_size=self.M)
        self.weight = torch.where(self.targets >= 0, self.weight, 0.0)
        self.weight /= self.weight.sum().clamp(min=1.0)


class NextId:
    """Table, one attention layer with a residual, and a norm before each of attention and loss."""

    def __init__(self, rows, D, heads, kv_heads, dtype="f32", seed=0):
        self.ctx = recd.Context(0)
        self.D, self.heads, self.kv_heads, self.d = D, heads, kv_heads, D // heads
        self.dtype = DTYPE[dtype]
        g = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, std):
            return torch.empty(*shape, device="cuda").normal_(0.0, std, generator=g)

        width = (heads + 2 * kv_heads) * self.d
        self.params = {"table": normal(rows, D, std=D ** -0.5), "w_qkv": normal(D, width, std=D ** -0.5),
                       "w_out": normal(heads * self.d, D, std=(heads * self.d) ** -0.5), "norm1": torch.ones(D, device="cuda"),
                       "bias1": torch.zeros(D, device="cuda"), "norm2": torch.ones(D, device="cuda"),
                       "bias2": torch.zeros(D, device="cuda")}
        self.squares = {n: torch.zeros_like(p) for n, p in self.params.items()}
        self.slopes = 2.0 ** (-8.0 * torch.arange(1, heads + 1, device="cuda", dtype=torch.float32) / heads)
        self.scale = 1.0                                                    # of the logits

    def how(self):
        return dict(scale=self.d ** -0.5, slopes=self.slopes, causal=True)

    def _heads(self, qkv):
        rows = qkv.view(qkv.shape[0], self.heads + 2 * self.kv_heads, self.d)
        return rows[:, :self.heads], rows[:, self.heads:self.heads + self.kv_heads], rows[:, self.heads + self.kv_heads:]

    def forward(self, lists, train=True):
        """Mean loss of the batch, and what the backward pass needs."""
        c, p, dt, M, D = self.ctx, self.params, self.dtype, lists.M, self.D
        new = lambda *shape, dtype=dt: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
        s = {"table": p["table"].to(dt), "w_qkv": p["w_qkv"].to(dt), "w_out": p["w_out"].to(dt)}
        s["emb"] = new(M, D)
        c.sequence_lookup_unique([s["table"]], lists.ids, lists.offsets, lists.feat_uoff, lists.U, s["emb"])
        s["h"], s["stats1"] = new(M, D), new(M, 2, dtype=torch.float32)
        c.layer_norm(s["emb"], p["norm1"], p["bias1"], EPS, s["h"], s["stats1"])
        s["qkv"] = s["h"] @ s["w_qkv"]
        q, k, v = self._heads(s["qkv"])
        s["out"], s["lse"] = new(M, self.heads, self.d), new(M, self.heads, dtype=torch.float32)
        c.list_attention(q, k, v, lists.offsets, lists.offsets, lists.longest, lists.longest, s["out"], s["lse"], **self.how())
        s["y"] = s["emb"] + s["out"].view(M, -1) @ s["w_out"]
        s["x"], s["stats2"] = new(M, D), new(M, 2, dtype=torch.float32)
        c.layer_norm(s["y"], p["norm2"], p["bias2"], EPS, s["x"], s["stats2"])
        s["loss"], s["logsum"] = new(M, dtype=torch.float32), new(M, dtype=torch.float32)
        s["mean_row"] = new(M, D, dtype=torch.float32) if train else None
        c.vocab_loss(s["x"], s["table"], lists.targets, self.scale, s["loss"], s["logsum"], s["mean_row"])
        return (s["loss"] * lists.weight).sum(), s

    def backward(self, lists, s):
        """Gradients by all parameters, in fp32."""
        c, p, dt, M, D = self.ctx, self.params, self.dtype, lists.M, self.D
        like = torch.empty_like
        grads = {n: like(p[n]) for n in ("norm1", "bias1", "norm2", "bias2")}
        # fp16 gradients are scaled up on the way
        up = 2.0 ** 14 if dt == torch.float16 else 1.0
        g_x, g_table = like(s["x"]), like(s["table"])
        c.vocab_loss_backward(s["x"], s["table"], lists.targets, self.scale, s["logsum"], s["mean_row"], lists.weight * up,
                              g_x, g_table)
        g_y = like(s["y"])
        c.layer_norm_backward(s["y"], p["norm2"], s["stats2"], g_x, g_y, grads["norm2"], grads["bias2"])
        grads["w_out"] = s["out"].view(M, -1).t() @ g_y
        g_out = (g_y @ s["w_out"].t()).view_as(s["out"])
        g_qkv = like(s["qkv"])
        c.list_attention_backward(*self._heads(s["qkv"]), lists.offsets, lists.offsets, lists.longest, lists.longest, s["out"],
                                  s["lse"], g_out, *self._heads(g_qkv), **self.how())
        grads["w_qkv"] = s["h"].t() @ g_qkv
        g_emb = like(s["emb"])
        c.layer_norm_backward(s["emb"], p["norm1"], s["stats1"], g_qkv @ s["w_qkv"].t(), g_emb, grads["norm1"], grads["bias1"])
        g_emb = (g_emb + g_y).float()
        # the rows' gradients, summed per table row: the unique lists are a batch of their own
        touched = torch.empty(max(M, 1), dtype=torch.int64, device="cuda")
        feat_roff = torch.empty(2, dtype=torch.int64, device="cuda")
        rows = torch.empty(max(M, 1), D, device="cuda")
        R = c.backward_sequence_dedup(1, lists.U, g_emb, lists.offsets, torch.arange(lists.U, dtype=torch.int32, device="cuda"),
                                      lists.feat_uoff, lists.ids, lists.offsets, [p["table"].shape[0]], lists.U, M,
                                      torch.empty_like(rows), touched, feat_roff, rows, want_count=True)
        grads["table"] = g_table.float().index_add_(0, touched[:R], rows[:R])
        return {n: g.float() / up for n, g in grads.items()}

    def step(self, lists, lr):
        loss, s = self.forward(lists)
        for n, g in self.backward(lists, s).items():
            self.squares[n] += g * g
            self.params[n] -= lr * g / (self.squares[n].sqrt() + 1e-10)     # Adagrad
        return loss

    def last_rows(self, lists, s):
        """Serving: the newest position of every list alone, against the keys and values that the list has so far."""
        q, k, v = self._heads(s["qkv"])
        some = lists.offsets.diff() > 0
        last = lists.offsets[1:][some] - 1
        offsets = torch.cat([lists.offsets[:1], lists.offsets[1:][some]])
        one = torch.arange(last.numel() + 1, device="cuda")
        out = torch.empty(last.numel(), self.heads, self.d, dtype=self.dtype, device="cuda")
        self.ctx.list_attention(q[last].contiguous(), k, v, one, offsets, 1, lists.longest, out, **self.how())
        return last, out


def batch(B, rows, longest, seed):
    """Lists of sessions of eight samples on average; ids by a power law, each next one near the one before."""
    w = synth.Workload("next_id", 1, B, 1, 8, "uniform", longest, 0.0, "zipf", 1.05, rows, 64, "f32")
    b = synth.make_batch(w, seed)
    start = np.repeat(b.values[b.offsets[:-1].clip(max=max(b.N - 1, 0))], np.diff(b.offsets)) if b.N else b.values
    at = np.arange(b.N) - np.repeat(b.offsets[:-1], np.diff(b.offsets))
    return torch.from_numpy((start * 7 + at * 3) % rows).cuda(), torch.from_numpy(b.offsets).cuda()


def main():
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--steps", type=int, default=50)
    a.add_argument("--dtype", choices=list(DTYPE), default="bf16")
    a.add_argument("--batch", type=int, default=2048)
    a.add_argument("--rows", type=int, default=20_000)
    a.add_argument("--longest", type=int, default=64)
    a.add_argument("--dim", type=int, default=128)
    a.add_argument("--heads", type=int, default=4)
    a.add_argument("--kv-heads", type=int, default=2)
    a = a.parse_args()
    model = NextId(a.rows, a.dim, a.heads, a.kv_heads, a.dtype)
    for i in range(a.steps):
        lists = Lists(model.ctx, *batch(a.batch, a.rows, a.longest, i % 8))
        loss = model.step(lists, 0.05)
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i}: loss {float(loss):.4f}, {lists.U} unique lists of {a.batch}, {lists.M} rows", flush=True)


if __name__ == "__main__":
    main()
