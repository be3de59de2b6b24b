"""The weight gradient at sizes that take each of its tiles, whole and with its tokens
split (test_wgrad_plan.py pins which), against a product in 64 bits.  Tolerance as
in test_gpu_ckpt.py: 2 (T + 8) 2^-24 of the sum of magnitudes, and the result's
rounding."""
import pytest

import train_ops_ref as ref
from train_ops_ref import BF16, F32
from wgrad_tiles import CASES

pytestmark = pytest.mark.gpu


def laid_out(x, pad, offset):
    """x on the device with rows `pad` apart, `offset` elements into a buffer of guards."""
    import torch
    rows, width = x.shape
    buf = torch.full((rows * (width + pad) + offset + 8,), ref.GUARD, dtype=x.dtype, device="cuda")
    view = buf[offset:offset + rows * (width + pad)].view(rows, width + pad)[:, :width]
    view.copy_(x)
    return view, buf


def guards_intact(view, buf, pad, offset):
    rows, width = view.shape
    whole = buf[offset:offset + rows * (width + pad)].view(rows, width + pad)
    ends = (buf[:offset] == ref.GUARD).all() and (buf[offset + rows * (width + pad):] == ref.GUARD).all()
    return bool(ends) and bool((whole[:, width:] == ref.GUARD).all())


@pytest.mark.parametrize("grad_dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("case", [c[0] for c in CASES], ids=str)
def test_wgrad(case, dtype, grad_dtype):
    import torch
    import paper_1909_08029_amd as rip
    rows, n, k, pad, offset = case
    print(f"case wgrad tiles {case} {dtype} -> {grad_dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows + 3 * n + k)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x = rand(rows, k) * 2.0 ** torch.randint(-6, 7, (rows, 1), generator=gen, device="cuda")
    ck = rip.rip_ckpt_pack(x)
    xk = rip.rip_ckpt_unpack(ck, F32).double()
    dy, _ = laid_out((rand(rows, n) * 1e-3).to(dtype), pad, offset)
    d = dy.double().t().contiguous()
    want, mag = d @ xk, d.abs() @ xk.abs()
    for accumulate in (False, True):
        grad, buf = laid_out(rand(n, k).to(grad_dtype), pad, offset)
        start = grad.double() * accumulate
        rip.rip_ckpt_wgrad(dy, ck, grad, accumulate=accumulate)
        full = want + start
        tol = 2 * (rows + 8) * 2.0 ** -24 * (mag + start.abs()) + ref.HALF_ULP[grad_dtype] * full.abs()
        off = (grad.double() - full).abs()
        bad = ~(off <= tol)
        assert not bad.any(), (int(bad.sum()), torch.nonzero(bad)[0].tolist(), float((off / tol).max()))
        assert guards_intact(grad, buf, pad, offset)
        if not accumulate:   # the same bits every time
            again = torch.full_like(grad, 7.0)
            rip.rip_ckpt_wgrad(dy, ck, again)
            assert torch.equal(again, grad)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("case", [(300, 700, 900), (257, 2901, 2899), (33, 5003, 4999)], ids=str)
def test_infinities_and_nans_stay_in_their_rows_and_columns(case, dtype):
    import torch
    import paper_1909_08029_amd as rip
    rows, n, k = case
    x = torch.ones(rows, k, device="cuda")
    x[3, 40], x[rows - 1, k - 1] = float("nan"), float("inf")   # their blocks of 32 columns
    bad = torch.zeros(k, dtype=torch.bool, device="cuda")
    bad[32:64], bad[(k - 1) // 32 * 32:] = True, True
    dy = torch.ones(rows, n, device="cuda", dtype=dtype)
    dy[5, 2], dy[rows - 1, n - 1] = float("inf"), float("nan")
    grad = rip.rip_ckpt_wgrad(dy, rip.rip_ckpt_pack(x), torch.empty(n, k, device="cuda"))
    assert torch.isnan(grad[:, bad]).all() and torch.isnan(grad[n - 1]).all()
    assert (grad[2, ~bad] == float("inf")).all()
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[2] = rest[n - 1] = False
    assert (grad[rest][:, ~bad] == rows).all()
