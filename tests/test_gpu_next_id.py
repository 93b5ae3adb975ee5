"""The next-id example: its loss and gradients, computed once per unique list, against those of the whole batch in 64
bits, its serving form against its own rows, and that training lowers the loss."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("next_id", os.path.join(ROOT, "examples", "next_id.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def whole_batch(model, values, offsets):
    """Mean loss over all rows of the batch (duplicates included) and its gradients, by autograd on the CPU."""
    p = {n: t.double().cpu().requires_grad_() for n, t in model.params.items()}
    H, G, d = model.heads, model.kv_heads, model.d
    norm = lambda x, w, b: torch.nn.functional.layer_norm(x, (model.D,), w, b, 1e-5)  # noqa: E731
    slopes = model.slopes.double().cpu()
    total, count = 0.0, 0
    o, values = offsets.tolist(), values.cpu()
    for a, b in zip(o, o[1:]):
        n = b - a
        if n < 2:
            continue
        ids = values[a:b]
        emb = p["table"][ids]
        qkv = (norm(emb, p["norm1"], p["bias1"]) @ p["w_qkv"]).view(n, H + 2 * G, d)
        i = torch.arange(n)
        far = (i[:, None] - i).abs()
        heads = []
        for h in range(H):
            k, v = qkv[:, H + h // (H // G)], qkv[:, H + G + h // (H // G)]
            z = qkv[:, h] @ k.t() * d ** -0.5 - slopes[h] * far
            heads.append(torch.softmax(z.masked_fill(i[:, None] < i, -float("inf")), 1) @ v)
        y = emb + torch.stack(heads, 1).reshape(n, -1) @ p["w_out"]
        z = norm(y, p["norm2"], p["bias2"])[:-1] @ p["table"].t()
        total = total + torch.nn.functional.cross_entropy(z, ids[1:], reduction="sum")
        count += n - 1
    loss = total / count
    loss.backward()
    return float(loss.detach()), {n: t.grad for n, t in p.items()}


# fp32 sums and exponents: 1e-5 of a gradient's length holds every one of them; 16-bit steps each round by 2^-9 or 2^-12
# of a value, some twenty of them one behind the other
@pytest.mark.parametrize("dtype,bar", [("f32", 2e-5), ("f16", 1e-2), ("bf16", 5e-2)])
def test_gradients_are_those_of_the_whole_batch(example, dtype, bar):
    model = example.NextId(300, 64, 4, 2, dtype, seed=1)
    values, offsets = example.batch(60, 300, 12, 3)
    lists = example.Lists(model.ctx, values, offsets)
    assert lists.U < 60
    loss, s = model.forward(lists)
    grads = model.backward(lists, s)
    want, ref = whole_batch(model, values, offsets)
    assert abs(float(loss) - want) < bar * want
    for n, g in grads.items():
        err = (g.double().cpu() - ref[n]).norm() / ref[n].norm()
        assert err < bar, (n, float(err))


@pytest.mark.parametrize("dtype,bar", [("f32", 1e-5), ("bf16", 8e-3)])
def test_a_new_position_alone_gives_what_it_gives_among_its_list(example, dtype, bar):
    model = example.NextId(500, 64, 4, 1, dtype, seed=2)
    lists = example.Lists(model.ctx, *example.batch(80, 500, 40, 5))
    _, s = model.forward(lists, train=False)
    last, out = model.last_rows(lists, s)
    want = s["out"][last].float()
    assert (out.float() - want).norm() < bar * want.norm()


def test_training_lowers_the_loss(example):
    model = example.NextId(2000, 64, 4, 2, "bf16", seed=3)
    losses = [float(model.step(example.Lists(model.ctx, *example.batch(256, 2000, 30, i % 3)), 0.05)) for i in range(30)]
    assert all(x == x for x in losses)
    assert sum(losses[-3:]) < 0.5 * sum(losses[:3])
