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


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("tokens,vocab", [(12, 50), (3000, 40), (150, 40000), (40, 1031)])
def test_offsets_out_of_order_across_pairs(tokens, vocab, dtype):
    """A token belongs to one sequence at most, whatever the offsets: the same bits as
    with the offsets' running maximum within the tokens.  Sequences of one round of
    a workgroup's threads and of several, thousands of pairs, and no tokens."""
    import torch
    import paper_1909_08029_amd as rip
    rng = np.random.default_rng(tokens)
    x = torch.from_numpy(rng.standard_normal((tokens, vocab)) * 2).to(dtype).cuda()
    t = torch.from_numpy(rng.integers(0, vocab, tokens)).cuda()
    third = tokens // 3
    wild = [[0, tokens, third, tokens // 2, tokens], [third, 0, tokens, -7, 2 * tokens],
            [tokens, 0, third, tokens, tokens], [0, third, 2 * third, third, tokens],
            rng.integers(-tokens, 2 * tokens, 9).tolist(), [-2 ** 31, 2 ** 31 - 1, 0, 0, third],
            [0] * 5, (np.sort(rng.integers(0, tokens + 1, 6001)) - rng.integers(0, 5, 6001)).tolist()]
    for o in wild:
        fit = np.maximum.accumulate(np.clip(o, 0, tokens))
        r = torch.from_numpy(rng.standard_normal(len(o) - 1).astype(np.float32)).cuda()
        out = []
        for offsets in (o, fit):
            grad = torch.full_like(x, 5.0)
            od = torch.from_numpy(np.asarray(offsets, np.int32)).cuda()
            got = rip.rip_pref_loss(x, t, od, r, 0.3, 0.1, grad=grad)
            assert torch.equal(od.cpu(), torch.from_numpy(np.asarray(offsets, np.int32)))
            out.append([a.clone() for a in (*got, grad)])
        for a, b in zip(*out):
            assert torch.equal(a, b)
        inside = np.zeros(tokens, bool)
        inside[fit[0]:fit[-1]] = True
        assert (ref.host(out[0][2])[~inside] == 0).all() and (ref.host(out[0][2])[inside] < 0).all()
    od = torch.from_numpy(np.array([3, -1, 2, 0, 9], np.int32)).cuda()
    r = torch.tensor([1.0, 2.0, 0.5, 0.25], device="cuda")
    loss, seq, logp = rip.rip_pref_loss(x[:0], t[:0], od, r, 0.5)
    want = np.mean(np.log1p(np.exp(-0.5 * np.array([1.0, -0.25]))))
    assert abs(float(loss) - want) < 1e-6 and (seq == 0).all() and logp.numel() == 0


def test_offsets_in_order_against_the_plain_form():
    """Backward offsets with the running maximum as the plain form takes them."""
    import torch
    import paper_1909_08029_amd as rip
    rng = np.random.default_rng(11)
    x, t, xh, targets, logp = policy_inputs(rng, 90, 333, F32)
    offsets = np.array([0, 40, 20, 30, 60, 50, 90])
    fit = np.maximum.accumulate(offsets)
    r = rng.standard_normal(6).astype(np.float32) - 100
    beta = float(np.float32(0.2))
    want = ref.pref_loss(xh, targets, fit, r.astype(np.float64), beta, 0.0)
    grad = torch.empty_like(x)
    loss, seq, got = rip.rip_pref_loss(x, t, torch.from_numpy(offsets.astype(np.int32)).cuda(),
                                       torch.from_numpy(r).cuda(), beta, grad=grad)
    d = delta(xh, 333)
    ref.close(ref.host(got), want["logp"], d + 2.0 ** -23 * np.abs(want["logp"]), "logp")
    count = np.diff(fit) * d
    ref.close(ref.host(seq), want["seq"], count + 2.0 ** -23 * np.abs(want["seq"]), "seq")
    dz = beta * 2 * count.sum()
    ref.close(ref.host(loss), want["loss"], dz + 2.0 ** -20 * (1 + abs(want["loss"])), "loss")
    check_grad(ref.host(grad), want, targets, dz + 2.0 ** -20, F32)


@pytest.mark.parametrize("scale", [1e-4, 3e-4, 1e-3, 1e-2, 0.3, 2.0])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("form", FORMS, ids=str)
def test_kl_near_its_zero(form, dtype, scale):
    """A policy close to its reference: K = e^d - d - 1 is about d^2 / 2.  Without the
    first term the loss is kl * sum of w K; K has a relative error of 2^-20 and that of
    logp (delta, and its rounding), which K's derivative and half its square carry on."""
    import torch
    import paper_1909_08029_amd as rip
    tokens, vocab = form
    rng = np.random.default_rng(tokens + vocab)
    x, t, xh, targets, logp = policy_inputs(rng, tokens, vocab, dtype)
    refp = (logp + scale * rng.choice([-1, 1], tokens) * (1 + rng.random(tokens))).astype(np.float32)
    w = (rng.random(tokens) + 0.1).astype(np.float32)
    zero = np.zeros(tokens, np.float32)
    old = logp.astype(np.float32)
    kl = float(np.float32(0.05))
    want = ref.policy_loss(xh, targets, old.astype(np.float64), zero.astype(np.float64),
                           w.astype(np.float64), refp.astype(np.float64), 0.2, 0.2, 0.0)
    d = refp.astype(np.float64) - want["logp"]
    k, slope = np.where(want["counted"], np.expm1(d) - d, 0), np.where(want["counted"], -np.expm1(d), 0)
    k = np.where(want["counted"] & (np.abs(d) < 0.05), d * d * (1 / 2 + d * (1 / 6 + d * (1 / 24 + d / 120))), k)
    cuda = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    grad = torch.empty_like(x)
    loss, _ = rip.rip_policy_loss(x, t, cuda(old), cuda(zero), cuda(w), cuda(refp), 0.2, 0.2, kl, grad=grad)
    off = delta(xh, vocab) + 2.0 ** -23 * np.abs(want["logp"])
    tol = kl * w * (2.0 ** -20 * k + off * np.abs(slope) + off ** 2 * np.exp(d))
    loss64 = (kl * w * k)[want["counted"]].sum()
    ref.close(ref.host(loss), loss64, tol[want["counted"]].sum() + 2.0 ** -24 * loss64, "loss")
    want["coef"] = kl * w * slope
    rel = np.where(want["counted"], off * np.exp(d) / np.maximum(np.abs(slope), 1e-30) + 2.0 ** -20, 0)
    want["grad"] = ref.logits_grad(want["coef"], want["counted"], want["soft"], targets)
    check_grad(ref.host(grad), want, targets, rel[:, None], dtype)


def test_kl_beside_a_large_first_term():
    """A KL term of 5e-9 a token is not lost beside a first term of 1: it moves the
    sum over tokens whose first terms cancel."""
    import torch
    import paper_1909_08029_amd as rip
    x = torch.zeros(64, 32, device="cuda")
    t = torch.zeros(64, dtype=torch.int64, device="cuda")
    lp = rip.rip_policy_loss(x, t, torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda"))[1]
    adv = torch.tensor([1.0, -1.0], device="cuda").repeat(32)
    refp = lp + 1e-4
    k = torch.expm1((refp - lp).double()) - (refp - lp).double()
    loss, _ = rip.rip_policy_loss(x, t, lp, adv, torch.ones(64, device="cuda"), refp, kl=1.0)
    assert abs(float(loss) - float(k.sum())) <= 2.0 ** -20 * float(k.sum())
