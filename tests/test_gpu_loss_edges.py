"""Losses at the ends of their inputs' ranges, in every form of their launches (a
row to a workgroup of 64, 256 or 512 threads, rows split over workgroups), against
the plain 64-bit forms.  Tolerances as in test_gpu_losses.py, whose helpers are
used.
"""
import numpy as np
import pytest

import train_ops_ref as ref
from test_gpu_losses import check_grad, delta
from train_ops_ref import BF16, F32

pytestmark = pytest.mark.gpu

FORMS = [  # tokens, vocab: 64, 256, 512 threads a row, three launches
    (40, 333), (24, 5003), (520, 20011), (12, 70001)]


def policy_inputs(rng, tokens, vocab, dtype):
    import torch
    x, _ = ref.device_matrix(rng.standard_normal((tokens, vocab)) * 3, dtype)
    targets = rng.integers(0, vocab, tokens)
    targets[rng.random(tokens) < 0.2] = -100
    targets[:3] = (0, 1, 2)   # these count
    xh = ref.host(x)
    return x, torch.from_numpy(targets).cuda(), xh, targets, ref.log_softmax_at(xh, targets)[0]


@pytest.mark.parametrize("kl", [0.0, 0.25])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("form", FORMS, ids=str)
def test_ratios_beyond_fp32(form, dtype, kl):
    """Tokens without an advantage or a weight add nothing, also where e^(logp -
    old_logp) passes fp32: the 64-bit form has them with an old_logp at which it
    does not."""
    import torch
    import paper_1909_08029_amd as rip
    tokens, vocab = form
    rng = np.random.default_rng(tokens + vocab)
    x, t, xh, targets, logp = policy_inputs(rng, tokens, vocab, dtype)
    old = (logp - np.log(rng.choice([0.4, 0.7, 1.0, 1.1, 1.35, 2.0], tokens))).astype(np.float32)
    adv = rng.standard_normal(tokens).astype(np.float32)
    weight = (rng.random(tokens) + 0.1).astype(np.float32)
    refp = (logp + rng.standard_normal(tokens) * 0.5).astype(np.float32)
    kind = rng.integers(0, 4, tokens)
    kind[:3] = (1, 2, 3)
    adv[kind == 1] = 0
    weight[kind >= 2] = 0
    adv[kind == 2] = -np.abs(adv[kind == 2])
    wild, wild_ref = old.copy(), refp.copy()
    wild[kind > 0] = rng.choice([-200, -1e30, -3.4e38, -np.inf], int((kind > 0).sum()))
    wild_ref[kind == 3] = rng.choice([500, -1e30, 3e38, np.nan], int((kind == 3).sum()))
    cuda = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    f = lambda v: float(np.float32(v))  # noqa: E731
    low, high = f(0.2), f(0.28)
    want = ref.policy_loss(xh, targets, old.astype(np.float64), adv.astype(np.float64),
                           weight.astype(np.float64), refp.astype(np.float64), low, high, kl)
    grad = torch.full_like(x, 3.0)
    loss, got = rip.rip_policy_loss(x, t, cuda(wild), cuda(adv), cuda(weight),
                                    cuda(wild_ref) if kl else None, low, high, kl, grad=grad)
    d = delta(xh, vocab)
    ref.close(ref.host(got), want["logp"], d + 2.0 ** -23 * np.abs(want["logp"]), "logp")
    r = np.exp(want["logp"] - old)
    e = np.exp(refp - want["logp"]) if kl else 0 * r
    err = weight * (r * np.abs(adv) + kl * (e + np.abs(refp - want["logp"]) + 1)) * (4 * d + 2.0 ** -20)
    ref.close(ref.host(loss), want["loss"], err[want["counted"]].sum() + 2.0 ** -22, "loss")
    rel = np.divide(err, np.abs(want["coef"]), out=np.zeros_like(err), where=want["coef"] != 0)
    check_grad(ref.host(grad), want, targets, rel[:, None], dtype)
    nothing = (kind >= 2) | ((kind == 1) & (kl == 0))
    assert (ref.host(grad)[nothing] == 0).all()
