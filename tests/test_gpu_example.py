"""The example that trains replicas with all the operators together: its
gradients against automatic differentiation of the same model in plain torch, and
a few steps of training."""
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


@pytest.mark.parametrize("loss", ["preference", "policy"])
def test_gradients(example, loss):
    """fp32 replica.  A block's step is below 2/127 of its largest magnitude, so the
    checkpoints hold activations within 1/127 of it, as independent errors, and the
    gated unit's product has those of two and its own: the gradients' relative error
    (norm of the difference over the norm) stays below 4/127.  Against the same
    formulas in 64 bits on the checkpoints' own values it is fp32's: sums of up to
    211 terms, four products in a row, 4 * 211 * 2^-24 of the magnitudes."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(4)
    m = example.Model(211, 48, 80, torch.float32, gen)
    ref = example.Model(211, 48, 80, torch.float32, gen)
    b = example.make_batch(m, ref, 5, 13, gen)
    value, _ = m.gradients(b, loss)

    p = {k: v.double().requires_grad_() for k, v in m.param.items()}
    x = p["embed"][b["ids"]] * 48 ** 0.5
    h = torch.nn.functional.silu(x @ p["gate"].t()) * (x @ p["up"].t())
    logits = (x + h @ p["down"].t()) @ p["out"].t()
    counted = b["targets"] >= 0
    logp = torch.log_softmax(logits, 1).gather(1, b["targets"].clamp(min=0)[:, None])[:, 0] * counted
    if loss == "preference":
        r = logp.view(10, 13).sum(1) - b["ref_seq"].double()
        want = -torch.nn.functional.logsigmoid(0.2 * (r[0::2] - r[1::2])).mean()
    else:
        adv, old = b["adv"].double(), b["ref"].double()
        ratio, d = (logp - old).exp(), old - logp
        gain = torch.minimum(ratio * adv, ratio.clamp(0.8, 1.2) * adv)
        want = (b["weight"].double() * (0.01 * (d.exp() - d - 1) - gain)).sum()
    logits.retain_grad()
    want.backward()
    want, dlogits = want.detach(), logits.grad
    assert abs(float(value) - float(want)) <= 1e-4 * (1 + abs(float(want)))
    for k in p:
        e = float((m.grad[k].double() - p[k].grad).norm() / p[k].grad.norm())
        assert e < 4 / 127, (k, e)

    from paper_1909_08029_amd import rip_ckpt_unpack, rip_gate_backward
    _, (ids, x8, g8, u8, y8) = m.forward(b["ids"])
    w = {k: v.detach() for k, v in p.items()}
    dy = dlogits @ w["out"]
    dh = dy @ w["down"]
    _, _, h8 = rip_gate_backward(dh.float(), g8, u8, hidden=True)
    kept = lambda c: rip_ckpt_unpack(c, torch.float32).double()  # noqa: E731
    g, u = kept(g8), kept(u8)
    s = torch.sigmoid(g)
    dg, du = dh * u * s * (1 + g * (1 - s)), dh * g * s
    dx = (dy + dg @ w["gate"] + du @ w["up"]) * 48 ** 0.5
    exact = {"out": dlogits.t() @ kept(y8), "down": dy.t() @ kept(h8), "gate": dg.t() @ kept(x8),
             "up": du.t() @ kept(x8), "embed": torch.zeros_like(w["embed"]).index_add_(0, ids, dx)}
    for k in exact:
        e = float((m.grad[k].double() - exact[k]).norm() / exact[k].norm())
        assert e < 4 * 211 * 2.0 ** -24, (k, e)


@pytest.mark.parametrize("loss,bf16", [("preference", False), ("preference", True), ("policy", False)])
def test_training(example, loss, bf16):
    history = example.train(replicas=4, steps=25, loss=loss, bf16=bf16, log=None)
    print(loss, bf16, history[0], history[-1], flush=True)
    assert all(v == v for v, _ in history)
    assert history[-1][0] < history[0][0] - 0.02
    assert history[-1][1] > 0.75
