"""Attention over more sequences than every workgroup puts in order by itself (1024): a
launch before makes the running maximum of the offsets, and tiles find their sequence in
it.  Every element against 64 bits, and calls with offsets out of order to the bit
against calls with the same list put in order."""
import random

import pytest

from attn_ref import Attention, cleaned
from test_gpu_attn import offsets, run, table, tensors

pytestmark = pytest.mark.gpu


def lists(n, seed, longest=3):
    """(q_offsets, k_offsets) of n sequences of 0 .. longest tokens, other lengths on each
    side; the first begins behind a few tokens of none."""
    rng = random.Random(seed)
    sides = [[4], [2]]
    for side in sides:
        for _ in range(n):
            side.append(side[-1] + rng.randint(0, longest))
    return sides


def disordered(at, total, seed):
    """Numbers out of order in every round of 1024, across its borders, and beyond both ends."""
    rng, bad = random.Random(seed), list(at)
    for i in (0, 1, 511, 1022, 1023, 1024, 1025, 2047, 2048, len(bad) - 2, len(bad) - 1):
        if i < len(bad):
            bad[i] = rng.choice([-7, 0, bad[i] // 2, bad[i] + 40, bad[min(i + 30, len(bad) - 1)]])
    if len(bad) > 1100:
        bad[1030:1060] = reversed(bad[1030:1060])
        bad[1090] = bad[1095] + 9       # a top that the next ones lie below
    bad[-40] = total + 1000 if seed % 2 else bad[-40]
    return bad


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sequences", [1025, 2300])
@pytest.mark.parametrize("causal", [True, False])
def test_two_lists(dtype, sequences, causal):
    qo, ko = lists(sequences, sequences)
    x = tensors(dtype, 2, 1, 16, qo[-1] + 3, ko[-1] + 6)
    got = run(*x, qo, ko, causal=causal)
    Attention(*x[:3], qo, ko, causal, dout=x[3]).check(got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sequences", [1024, 1025, 1500, 2300])
@pytest.mark.parametrize("seed", [1, 2])
@pytest.mark.parametrize("two", [False, True])
def test_out_of_order(dtype, sequences, seed, two):
    import paper_1909_08029_amd as rip
    import torch
    qo, ko = lists(sequences, 10 * sequences + seed)
    nq, nk = qo[-1] + 5, ko[-1] + 5 if two else qo[-1] + 5
    qo = disordered(qo, nq, seed)
    ko = disordered(ko, nk, seed + 3) if two else None
    assert qo != cleaned(qo, nq) and (ko is None or ko != cleaned(ko, nk))
    x = tensors(dtype, 4, 2, 16, nq, nk, seed=seed)
    args = dict(causal=False, bias=table(5, 4), buckets=rip.RelBuckets([-2, -1, 0, 2], [4, 1, 0, 2, 3]))
    got = run(*x, qo, ko, **args)
    want = run(*x, cleaned(qo, nq), None if ko is None else cleaned(ko, nk), **args)
    for name, t in got.items():
        assert torch.equal(t, want[name]), name
    if sequences == 1500 and seed == 1:    # (the reference loops over sequences)
        rel = dict(bias=args["bias"], starts=args["buckets"].starts, rows=args["buckets"].rows)
        Attention(*x[:3], qo, ko, False, dout=x[3], **rel).check(got)


def test_a_few_long_ones_among_many():
    """Sequences of many tiles at both ends of the list and across its border of 1024."""
    qo, at = [0], 0
    for i in range(1400):
        at += {3: 300, 1023: 700, 1024: 150, 1399: 411}.get(i, i % 2)
        qo.append(at)
    for dtype in ("f32", "bf16"):
        x = tensors(dtype, 2, 2, 64, at, at)
        Attention(*x[:3], qo, dout=x[3]).check(run(*x, qo))
    import torch
    torch.cuda.synchronize()
