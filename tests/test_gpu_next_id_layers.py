"""The next-id example with its feed-forward block, dropout and answers: gradients against autograd in 64 bits on the CPU, with the masks
made again from their numbers, and the answers against the logits of its own rows."""
import importlib.util
import os

import pytest
import torch

from tests import layers_util as lu

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("next_id", os.path.join(ROOT, "examples", "next_id.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def reference(model, lists):
    """Loss and gradients over the unique lists, each as often as the batch holds it."""
    p = {n: t.double().cpu().requires_grad_() for n, t in model.params.items()}
    H, G, d, D = model.heads, model.kv_heads, model.d, model.D
    norm = lambda x, w, b: torch.nn.functional.layer_norm(x, (D,), w, b, 1e-5)  # noqa: E731

    def drop(x, which):
        if not model.dropout:
            return x
        mask = lu.keep(*x.shape, model.dropout, model.seed, 3 * model.steps + which).double()
        return x * mask * 65536.0 / (65536 - lu.cut(model.dropout))

    slopes = model.slopes.double().cpu()
    o, ids = lists.offsets.tolist(), lists.ids.cpu()
    emb = p["table"][ids]
    qkv = (norm(emb, p["norm1"], p["bias1"]) @ p["w_qkv"]).view(len(ids), H + 2 * G, d)
    out = []
    for a, b in zip(o, o[1:]):
        i = torch.arange(b - a)
        heads = []
        for h in range(H):
            k, v = qkv[a:b, H + h // (H // G)], qkv[a:b, H + G + h // (H // G)]
            z = qkv[a:b, h] @ k.t() * d ** -0.5 - slopes[h] * (i[:, None] - i).abs()
            heads.append(torch.softmax(z.masked_fill(i[:, None] < i, -float("inf")), 1) @ v)
        out.append(torch.stack(heads, 1).reshape(b - a, -1))
    y = emb + drop(torch.cat(out) @ p["w_out"], 0)
    if model.hidden:
        up = torch.nn.functional.gelu(norm(y, p["norm3"], p["bias3"]) @ p["w_up"].t() + p["bias_up"])
        y = y + drop(drop(up, 1) @ p["w_down"].t() + p["bias_down"], 2)
    z = norm(y, p["norm2"], p["bias2"]) @ p["table"].t()
    loss = torch.nn.functional.cross_entropy(z, lists.targets.cpu(), ignore_index=-1, reduction="none")
    total = (loss * lists.weight.double().cpu()).sum()
    total.backward()
    return float(total.detach()), {n: t.grad for n, t in p.items()}


# (the bars as without the block: fp32 sums and exponents, and some thirty 16-bit steps one behind the other)
@pytest.mark.parametrize("dtype,bar", [("f32", 2e-5), ("f16", 1e-2), ("bf16", 5e-2)])
@pytest.mark.parametrize("hidden,dropout", [(136, 0.0), (136, 0.25), (0, 0.5)])
def test_gradients(example, dtype, bar, hidden, dropout):
    model = example.NextId(300, 64, 4, 2, dtype, seed=1, hidden=hidden, dropout=dropout)
    for step in range(2):                                                  # (another step has other masks)
        lists = example.Lists(model.ctx, *example.batch(60, 300, 12, 3 + step))
        want, ref = reference(model, lists)
        loss, s = model.forward(lists)
        grads = model.backward(lists, s)
        assert grads.keys() == ref.keys()
        assert abs(float(loss) - want) < bar * want
        for n, g in grads.items():
            err = (g.double().cpu() - ref[n]).norm() / ref[n].norm()
            assert err < bar, (n, float(err))
        model.steps += 1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_answers_are_those_of_the_last_rows(example, dtype):
    model = example.NextId(500, 64, 4, 2, dtype, seed=2, hidden=72, dropout=0.3)
    lists = example.Lists(model.ctx, *example.batch(80, 500, 40, 5))
    ids, logp, entropy = model.answers(lists, 7)
    _, s = model.forward(lists, train=False)
    last = (lists.offsets[1:] - 1)[lists.offsets.diff() > 0]
    ref, want = lu.answers_ref(s["x"][last].cpu(), s["table"].cpu(), model.scale, torch.zeros(len(last), dtype=torch.int64), 7)
    assert torch.equal(ids.cpu(), want)
    assert ((logp.double().cpu() - ref["top_logp"][0]).abs() <= ref["top_logp"][1] + 1e-6 * ref["top_logp"][0].abs()).all()
    assert ((entropy.double().cpu() - ref["entropy"][0]).abs() <= ref["entropy"][1] + 1e-6 * ref["entropy"][0].abs()).all()


def test_training_runs_as_a_command(example, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["next_id.py", "--steps", "3", "--batch", "64", "--rows", "500", "--longest", "12", "--dim", "64",
                                     "--hidden", "128", "--dropout", "0.1"])
    example.main()
    said = capsys.readouterr().out
    assert "step 2" in said and "next of list 0" in said
