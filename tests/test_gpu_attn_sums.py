"""The softmax's sum over long sequences: its error does not grow with their length."""
import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("dtype,dim,keys", [("f32", 64, 200003), ("bf16", 64, 200003), ("bf16", 128, 100000),
                                            ("f32", 160, 40000)])
@pytest.mark.parametrize("below", [3.0, 5.0])
def test_equal_scores_below_a_larger_one(dtype, dim, keys, below):
    """One key of score 0, all others at -below; queries enough that a workgroup takes the
    whole sequence or half of it: the log-sum is log(1 + (keys - 1) e^-below).

    Scores are exact (one product that is not 0).  Errors in units of U = 2^-24, half a step:
      argument of e^x   x log2(e), of at most 8, rounded from a rounded scale: 2 * 8 * ln 2 < 12
      2^x               a step: 2
      a lane's sum      trees of at most 16 terms to a tile, and their compensated sum: 16 + 4
      its two halves    1
      log2, the sum with the reference 0, and ln 2 rounded and multiplied, of the result:
                        (2 + 1 + 1 + 1) |lse|
    """
    import torch
    import paper_1909_08029_amd as rip
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    queries, heads = 1300, 32
    q = torch.zeros(queries, heads, dim, device="cuda", dtype=t)
    q[..., dim - 1] = 1
    k = torch.zeros(keys, 1, dim, device="cuda", dtype=t)
    k[1:, 0, dim - 1] = -below
    at = lambda n: torch.tensor([0, n], dtype=torch.int32, device="cuda")  # noqa: E731
    out, kept = rip.rip_attn_forward(q, k, k, at(queries), at(keys), causal=False, scale=1.0)
    want = math.log1p((keys - 1) * math.exp(-below))
    bound = (35 + 5 * want) * U
    worst = float((kept.lse.double() - want).abs().max())
    assert worst <= bound, (worst, bound)
