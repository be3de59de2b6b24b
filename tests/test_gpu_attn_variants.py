"""Every variant of the attention kernels (widths, waves, whole and split, with and
without a bias) at the sizes of attn_plans.py, each element within its bound."""
import pytest

from attn_plans import SHAPES, WIDTHS
from attn_ref import Attention
from test_gpu_attn import offsets, run, table, tensors

pytestmark = pytest.mark.gpu


def packed(n, length):
    """Offsets of n sequences of about `length` tokens (exactly n * length in all)."""
    if n == 1 or length < 8:
        return [i * length for i in range(n + 1)]
    return [i * length + (i % 2) * (length // 4) for i in range(n)] + [n * length]


@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("shape", SHAPES)
def test_variant(shape, width, dtype, biased):
    import paper_1909_08029_amd as rip
    n, q, k, heads, group, causal = SHAPES[shape]
    x = tensors(dtype, heads, heads // group, WIDTHS[width], n * q, n * k)
    qo, ko = packed(n, q), packed(n, k)
    more, rel = {}, {}
    if biased:
        b = rip.RelBuckets.log(16, 60, not causal)
        more = dict(bias=table(16, heads), buckets=b)
        rel = dict(bias=more["bias"], starts=b.starts, rows=b.rows)
    got = run(*x, qo, None if q == k else ko, causal, **more)
    if heads > 8:                                    # some of them against the definition
        for first in (0, heads - 2):
            h = slice(first, first + 2)
            part = dict(rel, bias=rel["bias"][:, h]) if biased else {}
            Attention(*[t[:, h] for t in x[:3]], qo, ko, causal, dout=x[3][:, h], **part).check(
                {n: (t[h] if n == "lse" else t[:, h]) for n, t in got.items()})
    else:
        Attention(*x[:3], qo, ko, causal, dout=x[3], **rel).check(got)
    if biased:                                       # a forward pass alone: p rounded once
        out, kept = rip.rip_attn_forward(*x[:3], offsets(qo), None if q == k else offsets(ko), causal,
                                         keep=False, **more)
        assert kept is None
        Attention(x[0][:, :group], x[1][:, :1], x[2][:, :1], qo, ko, causal, low=False,
                  **dict(rel, bias=rel["bias"][:, :group])).check(dict(out=out[:, :group]))
