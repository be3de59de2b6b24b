"""The example's model with attention and its AdamW update: all the operators together,
gradients against automatic differentiation of the same model in 64 bits."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location(
        "preference_replicas", os.path.join(ROOT, "examples", "preference_replicas.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_gradients(example):
    """fp32.  The checkpoints hold the linear layers' inputs within 1/127 of them, as
    independent errors (a block's step is below 2/127 of its largest magnitude), and the
    gated unit's product has those of its two inputs and its own: the gradients'
    relative error stays below 4/127, as without attention, whose own errors are
    fp32's."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(4)
    m = example.AttentionModel(211, 48, 80, torch.float32, gen)
    ref = example.AttentionModel(211, 48, 80, torch.float32, gen)
    b = example.make_batch(m, ref, 5, 13, gen)
    value, _ = m.gradients(b, "preference")

    p = {k: v.double().requires_grad_() for k, v in m.param.items()}
    x = p["embed"][b["ids"]] * 48 ** 0.5
    q, k, v = ((x @ p["qkv"].t())[:, 48 * i:48 * (i + 1)].view(10, 13, 4, 12).transpose(1, 2) for i in range(3))
    rel = torch.arange(13, device="cuda")[None, :] - torch.arange(13, device="cuda")[:, None]
    row = torch.zeros_like(rel) + m.buckets.rows[0]
    for start, r in zip(m.buckets.starts, m.buckets.rows[1:]):
        row[rel >= start] = r
    scores = q @ k.transpose(2, 3) / 12 ** 0.5 + p["bias"][row].permute(2, 0, 1)
    a = torch.softmax(scores.masked_fill(rel > 0, -torch.inf), 3) @ v
    z = x + a.transpose(1, 2).reshape(130, 48) @ p["proj"].t()
    h = torch.nn.functional.silu(z @ p["gate"].t()) * (z @ p["up"].t())
    logits = (z + h @ p["down"].t()) @ p["out"].t()
    counted = b["targets"] >= 0
    logp = torch.log_softmax(logits, 1).gather(1, b["targets"].clamp(min=0)[:, None])[:, 0] * counted
    r = logp.view(10, 13).sum(1) - b["ref_seq"].double()
    want = -torch.nn.functional.logsigmoid(0.2 * (r[0::2] - r[1::2])).mean()
    want.backward()
    want = want.detach()
    assert abs(float(value) - float(want)) <= 1e-4 * (1 + abs(float(want)))
    for name in p:
        e = float((m.grad[name].double() - p[name].grad).norm() / p[name].grad.norm())
        assert e < 4 / 127, (name, e)


@pytest.mark.parametrize("loss,bf16,adamw", [("preference", False, 0), ("preference", True, 8),
                                             ("policy", False, 32), ("policy", True, 32)])
def test_runs(example, loss, bf16, adamw):
    history = example.train(replicas=3, steps=4, loss=loss, bf16=bf16, attention=True, adamw=adamw,
                            log=None)
    print(loss, bf16, adamw, history[0], history[-1], flush=True)
    assert len(history) == 4 and all(v == v and 0 <= share <= 1 for v, share in history)
