#!/usr/bin/env python3
"""Preference (or policy) training of small language-model replicas on one GPU.

    python examples/preference_replicas.py [--replicas 4] [--steps 40]
                                           [--loss preference|policy] [--bf16]
                                           [--attention] [--adamw 32|8]

Every step each replica runs its forward and backward pass on its own batch
(``Model.gradients``) and writes its gradients into the buffers registered with
``rip.Replicas``; then ``rip.rip_step`` makes the groups of the step, updates the
replicas and averages the groups in one launch.

The model is one gated feed-forward block between an embedding and a vocabulary
projection.  Its backward pass keeps three checkpoints of 8 bits (the block's
input, the gated unit's two inputs) and one made during the backward pass (the
gated unit's output) in place of the activations, and the logits' gradient
overwrites the logits.

With ``--attention`` a layer of causal attention with a learned relative position bias
comes before the block (``AttentionModel``).  With ``--adamw`` the local update is AdamW
with moments of 32 or 8 bits, and rip_preduce averages the groups.

The data are synthetic: a sequence follows a fixed rule (chosen) or does not
(rejected, or a negative advantage), and the first token is its prompt.
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_1909_08029_amd as rip  # noqa: E402

IGNORE = -100


class Model:
    """Parameters and gradients of one replica as views of two flat buffers."""

    def __init__(self, vocab: int, width: int, inner: int, dtype, generator):
        self.shapes = {"embed": (vocab, width), "gate": (inner, width), "up": (inner, width),
                       "down": (width, inner), "out": (vocab, width)}
        self.vocab, self.width, self.dtype = vocab, width, dtype
        self.param = {k: (torch.randn(s, generator=generator, device="cuda") / s[1] ** 0.5).to(dtype)
                      for k, s in self.shapes.items()}
        self.param["out"] *= 0.5
        self.grad = {k: torch.zeros_like(p) for k, p in self.param.items()}

    def segments(self, of):
        """The layer tensors in a fixed order, as rip.Replicas takes them."""
        return [of[k].view(-1) for k in self.shapes]

    def forward(self, ids, offsets=None):
        """(logits, what the backward pass needs); ``offsets``: where the sequences of
        the packed ids begin."""
        p = self.param
        x = rip.rip_embed_lookup(p["embed"], ids, self.width ** 0.5)
        x8 = rip.rip_ckpt_pack(x)
        h, gate8, up8 = rip.rip_gate_forward(x @ p["gate"].t(), x @ p["up"].t())
        y = x + h @ p["down"].t()
        return y @ p["out"].t(), (ids, x8, gate8, up8, rip.rip_ckpt_pack(y))

    def backward(self, dlogits, kept):
        """Fills the gradient buffers from the logits' gradient."""
        ids, x8, gate8, up8, y8 = kept
        p, g = self.param, self.grad
        rip.rip_ckpt_wgrad(dlogits, y8, g["out"])
        dy = dlogits @ p["out"]
        dgate, dup, h8 = rip.rip_gate_backward(dy @ p["down"], gate8, up8, hidden=True)
        rip.rip_ckpt_wgrad(dy, h8, g["down"])
        rip.rip_ckpt_wgrad(dgate, x8, g["gate"])
        rip.rip_ckpt_wgrad(dup, x8, g["up"])
        dx = dy + dgate @ p["gate"] + dup @ p["up"]
        rip.rip_embed_grad(dx, ids, g["embed"], self.width ** 0.5)

    def gradients(self, batch, loss: str):
        """The loss of a batch; its gradients are in ``grad`` afterwards."""
        logits, kept = self.forward(batch["ids"], batch["offsets"])
        if loss == "preference":
            value, seq, _ = rip.rip_pref_loss(logits, batch["targets"], batch["offsets"],
                                              batch["ref_seq"], beta=0.2, grad=logits)
            r = seq - batch["ref_seq"]
            better = (r[0::2] > r[1::2]).float().mean()
        else:
            value, logp = rip.rip_policy_loss(logits, batch["targets"], batch["ref"], batch["adv"],
                                              batch["weight"], batch["ref"], 0.2, 0.2, 0.01,
                                              grad=logits)
            better = ((logp - batch["ref"]) * batch["adv"] > 0).float().sum() / \
                (batch["adv"] != 0).sum()
        self.backward(logits, kept)
        return value, better


class AttentionModel(Model):
    """A layer of attention before the block.  q, k, v and the gradients of all three
    lie side by side in the rows of one projection; the bias is a table of buckets by
    distance."""

    def __init__(self, vocab: int, width: int, inner: int, dtype, generator, heads: int = 4,
                 buckets: int = 8, max_distance: int = 16):
        super().__init__(vocab, width, inner, dtype, generator)
        self.heads, self.dim = heads, width // heads
        self.buckets = rip.RelBuckets.log(buckets, max_distance, bidirectional=False)
        more = {"qkv": (3 * width, width), "proj": (width, width), "bias": (buckets, heads)}
        for k, shape in more.items():
            self.param[k] = (torch.randn(shape, generator=generator, device="cuda")
                             * (0.1 if k == "bias" else width ** -0.5)).to(dtype)
            self.grad[k] = torch.zeros_like(self.param[k])
        self.shapes.update(more)

    def _split(self, qkv):
        return [part.unflatten(1, (self.heads, self.dim)) for part in qkv.split(self.width, 1)]

    def forward(self, ids, offsets=None):
        p = self.param
        x = rip.rip_embed_lookup(p["embed"], ids, self.width ** 0.5)
        x8 = rip.rip_ckpt_pack(x)
        qkv = x @ p["qkv"].t()
        a, sums = rip.rip_attn_forward(*self._split(qkv), offsets, bias=p["bias"], buckets=self.buckets)
        a8 = rip.rip_ckpt_pack(a.flatten(1))
        z = x + a.flatten(1) @ p["proj"].t()
        z8 = rip.rip_ckpt_pack(z)
        h, gate8, up8 = rip.rip_gate_forward(z @ p["gate"].t(), z @ p["up"].t())
        y = z + h @ p["down"].t()
        kept = (ids, offsets, x8, qkv, a, sums, a8, z8, gate8, up8, rip.rip_ckpt_pack(y))
        return y @ p["out"].t(), kept

    def backward(self, dlogits, kept):
        ids, offsets, x8, qkv, a, sums, a8, z8, gate8, up8, y8 = kept
        p, g = self.param, self.grad
        rip.rip_ckpt_wgrad(dlogits, y8, g["out"])
        dy = dlogits @ p["out"]
        dgate, dup, h8 = rip.rip_gate_backward(dy @ p["down"], gate8, up8, hidden=True)
        rip.rip_ckpt_wgrad(dy, h8, g["down"])
        rip.rip_ckpt_wgrad(dgate, z8, g["gate"])
        rip.rip_ckpt_wgrad(dup, z8, g["up"])
        dz = dy + dgate @ p["gate"] + dup @ p["up"]
        rip.rip_ckpt_wgrad(dz, a8, g["proj"])
        dqkv = torch.empty_like(qkv)
        dq, dk, dv = self._split(dqkv)
        rip.rip_attn_backward((dz @ p["proj"]).view_as(a), *self._split(qkv), a, sums, offsets,
                              bias=p["bias"], buckets=self.buckets, dbias=g["bias"],
                              dq=dq, dk=dk, dv=dv)
        rip.rip_ckpt_wgrad(dqkv, x8, g["qkv"])
        rip.rip_embed_grad(dz + dqkv @ p["qkv"], ids, g["embed"], self.width ** 0.5)


def make_batch(model: Model, reference: Model, pairs: int, length: int, generator):
    """Pairs of sequences packed one after another, with the reference's
    log-probabilities."""
    vocab, n = model.vocab, 2 * pairs * length
    seq = torch.randint(0, vocab, (2 * pairs, length + 1), generator=generator, device="cuda")
    for t in range(length):  # the rule that chosen sequences follow
        seq[0::2, t + 1] = (5 * seq[0::2, t] + 1) % vocab
    ids, targets = seq[:, :-1].reshape(n).contiguous(), seq[:, 1:].reshape(n).contiguous()
    targets[::length] = IGNORE
    batch = dict(ids=ids, targets=targets,
                 offsets=torch.arange(2 * pairs + 1, device="cuda", dtype=torch.int32) * length)
    logits, _ = reference.forward(ids, batch["offsets"])
    _, batch["ref_seq"], batch["ref"] = rip.rip_pref_loss(
        logits, targets, batch["offsets"], torch.zeros(2 * pairs, device="cuda"))
    counted = targets != IGNORE
    sign = torch.ones(2 * pairs, length, device="cuda")
    sign[1::2] = -1
    batch["adv"] = sign.view(n) * counted
    batch["weight"] = counted / counted.sum().float()
    return batch


def train(replicas=4, steps=40, loss="preference", bf16=False, vocab=499, width=64, inner=176,
          pairs=8, length=24, lr=None, seed=0, log=print, attention=False, adamw=0):
    """Trains; returns the mean loss and the share of better pairs (tokens) of
    each step.  ``adamw``: bits of AdamW's moments, 0 for SGD."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.bfloat16 if bf16 else torch.float32
    kind = AttentionModel if attention else Model
    first = kind(vocab, width, inner, dtype, gen)
    models = [first] + [kind(vocab, width, inner, dtype, gen) for _ in range(replicas - 1)]
    reference = kind(vocab, width, inner, dtype, gen)
    for m in models[1:] + [reference]:  # one start, and a frozen copy of it
        for k, p in m.param.items():
            p.copy_(first.param[k])
    rep = rip.Replicas([m.segments(m.param) for m in models], [m.segments(m.grad) for m in models])
    sched = rip.Scheduler(replicas, rip.SCHED_GD, seed=seed, kmin=2, kmax=min(4, max(2, replicas)))
    state = rip.AdamwState.zeros(rep, adamw) if adamw else None
    lr = lr or (1e-2 if adamw else 0.5 if loss == "preference" else 2.0)
    history = []
    for step in range(steps):
        out = [m.gradients(make_batch(m, reference, pairs, length, gen), loss) for m in models]
        if adamw:
            active, groups = rip.rip_schedule_groups(sched, step)
            rip.rip_adamw_step(state, active, step + 1, lr, seed=seed)
            rip.rip_preduce(rep, groups)
        else:
            rip.rip_step(sched, rep, step, lr=lr)
        value, better = (float(sum(x[i] for x in out)) / replicas for i in (0, 1))
        history.append((value, better))
        if log and (step % 5 == 0 or step == steps - 1):
            log(f"step {step:3d}  loss {value:.4f}  better {better:.3f}")
    return history


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--replicas", type=int, default=4)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--loss", choices=["preference", "policy"], default="preference")
    ap.add_argument("--bf16", action="store_true")
    ap.add_argument("--attention", action="store_true")
    ap.add_argument("--adamw", type=int, choices=[0, 8, 32], default=0, help="bits of the moments")
    args = ap.parse_args()
    if not torch.cuda.is_available():
        raise SystemExit("needs a GPU")
    train(args.replicas, args.steps, args.loss, args.bf16, attention=args.attention, adamw=args.adamw)


if __name__ == "__main__":
    main()
