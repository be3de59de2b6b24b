"""The gated unit's backward pass at magnitudes whose products leave fp32, against the
plain 64-bit form (tolerances as in test_gpu_ckpt.py)."""
import numpy as np
import pytest

import train_ops_ref as ref
from test_gpu_ckpt import GATE_TOL, packed
from train_ops_ref import BF16, F32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_products_beyond_fp32_on_the_way(dtype):
    """dh * up passes fp32, dgate does not: the sigmoid between them is small."""
    import torch
    import paper_1909_08029_amd as rip
    gate = np.repeat(np.array([[-50.0], [-30.0], [-300.0], [-20.0]]), 40, axis=1)
    up = np.repeat(np.array([[1e20], [-1e25], [1e30], [3e37]]), 40, axis=1)
    dh = np.repeat(np.array([[1e25], [1e20], [1e20], [-2e3]]), 40, axis=1)
    (g, _), (u, _), (d, _) = (ref.device_matrix(x, dtype) for x in (gate, up, dh))
    _, g8, u8 = rip.rip_gate_forward(g, u)
    dgate, dup = rip.rip_gate_backward(d, g8, u8)
    gk, uk, dd = ref.unpack(*packed(g8), 40), ref.unpack(*packed(u8), 40), ref.host(d)
    s = ref.sigmoid(gk)
    want = dd * uk * s * (1 + gk * (1 - s))
    assert (np.abs(dd * uk) > 3.5e38).all() and (np.abs(want) < 3e38).all()
    # e^-300 is 0 in fp32
    tol = (GATE_TOL + ref.HALF_ULP[dtype]) * np.abs(want) + np.where(gk < -100, np.abs(want), 0)
    ref.close(ref.host(dgate), want, tol, "dgate")
    want = dd * gk * s
    tol = (GATE_TOL + ref.HALF_ULP[dtype]) * np.abs(want) + np.where(gk < -100, np.abs(want), 0)
    ref.close(ref.host(dup), want, tol, "dup")
    assert torch.isfinite(dgate).all()
