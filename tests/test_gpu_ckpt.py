"""8-bit activation checkpoints, the gated unit and the weight gradient that use
them, against plain 64-bit forms.

Tolerances.  Packing and unpacking are exact (integers and powers of two).  The
gated unit's sigmoid is good to 8 units in the last place and every formula here
adds a few roundings: 2^-20 of the terms' magnitudes, and the result's rounding.
A weight gradient's products are exact and its sum of T terms is fp32:
2 (T + 8) 2^-24 of the sum of magnitudes, and the result's rounding.
"""
import numpy as np
import pytest

import train_ops_ref as ref
from train_ops_ref import BF16, F32

pytestmark = pytest.mark.gpu

SHAPES = [  # rows, width, pad, offset
    (1, 1, 0, 0), (1, 31, 0, 0), (3, 32, 0, 1), (2, 33, 3, 0), (5, 100, 0, 3), (17, 1031, 1, 1),
    (64, 256, 0, 0), (1, 5504, 0, 0), (130, 40, 8, 5)]


def values(rng, rows, width):
    """Magnitudes from 2^-140 to 2^126, blocks of zeros, of one value, of ties."""
    x = rng.standard_normal((rows, width))
    x *= 2.0 ** rng.choice([-150, -130, -126, -20, -3, 0, 4, 60, 120], (rows, 1))
    for r in range(0, rows, 3):
        x[r, :32] = 0
    for r in range(1, rows, 3):
        x[r, -5:] = 1.984375 * 2.0 ** (r % 7)      # 127 steps exactly, the largest of its block
    if rows > 2:
        x[2, :] = np.arange(width) % 64 + 64.5     # ties
    with np.errstate(over="ignore"):
        return x.astype(np.float32)


def packed(t):
    return t.codes.cpu().numpy(), t.exps.cpu().numpy()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("rows,width,pad,offset", SHAPES)
def test_pack_and_unpack(rows, width, pad, offset, dtype):
    import torch
    import paper_1909_08029_amd as rip
    rng = np.random.default_rng(rows * 100 + width)
    x, _ = ref.device_matrix(values(rng, rows, width), dtype, pad, offset)
    got = rip.rip_ckpt_pack(x)
    codes, exps = ref.pack(x.float().cpu().numpy())
    assert np.array_equal(got.codes.cpu().numpy(), codes)
    assert np.array_equal(got.exps.cpu().numpy(), exps)
    want = ref.unpack(codes, exps, width)
    for out_type in (F32, BF16):   # exact in both
        out, buf = ref.device_matrix(np.zeros((rows, width)), out_type, pad, offset)
        rip.rip_ckpt_unpack(got, out=out)
        assert np.array_equal(ref.host(out), want)
        assert ref.guards_intact(out, buf)
    # what a checkpoint stands for packs to itself
    again = rip.rip_ckpt_pack(rip.rip_ckpt_unpack(got, F32))
    assert torch.equal(rip.rip_ckpt_unpack(again, F32), rip.rip_ckpt_unpack(got, F32))


def test_blocks_with_infinities_and_nans():
    import torch
    import paper_1909_08029_amd as rip
    x = torch.ones(3, 70, device="cuda")
    x[0, 40], x[1, 69], x[1, 0] = float("nan"), float("inf"), float("-inf")
    for dtype in (F32, BF16):
        c = rip.rip_ckpt_pack(x.to(dtype))
        assert c.exps.tolist() == [[121, 255, 121], [255, 121, 255], [121, 121, 121]]
        y = rip.rip_ckpt_unpack(c)
        bad = torch.isnan(y)
        assert bad[0, 32:64].all() and bad[1, :32].all() and bad[1, 64:].all() and int(bad.sum()) == 70
        assert (y[~bad] == 1).all()


def test_the_largest_numbers_do_not_overflow():
    import torch
    import paper_1909_08029_amd as rip
    for dtype in (F32, BF16):
        big = torch.full((1, 32), torch.finfo(dtype).max, device="cuda", dtype=dtype)
        y = rip.rip_ckpt_unpack(rip.rip_ckpt_pack(big), F32)
        assert torch.isfinite(y).all() and (y == 127 * 2.0 ** 121).all()


GATE_TOL = 2.0 ** -20


def gate_inputs(rng, rows, width, dtype, pad, offset, sigma=2.0):
    g, _ = ref.device_matrix(rng.standard_normal((rows, width)) * sigma, dtype, pad, offset)
    u, _ = ref.device_matrix(rng.standard_normal((rows, width)), dtype, pad, offset)
    d, _ = ref.device_matrix(rng.standard_normal((rows, width)) * 1e-2, dtype, pad, offset)
    return g, u, d


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("rows,width,pad,offset", SHAPES)
def test_gate(rows, width, pad, offset, dtype):
    import torch
    import paper_1909_08029_amd as rip
    rng = np.random.default_rng(rows + width)
    for sigma in (2.0, 40.0):
        g, u, d = gate_inputs(rng, rows, width, dtype, pad, offset, sigma)
        h, hbuf = ref.device_matrix(np.zeros((rows, width)), dtype, pad, offset)
        _, g8, u8 = rip.rip_gate_forward(g, u, out=h)
        for x, c in ((g, g8), (u, u8)):
            codes, exps = ref.pack(x.float().cpu().numpy())
            assert np.array_equal(packed(c)[0], codes) and np.array_equal(packed(c)[1], exps)
        gd, ud = ref.host(g), ref.host(u)
        want = gd * ref.sigmoid(gd) * ud
        # far below, e^-80 stands for e^g: a difference of less than 1e-30
        tol = (GATE_TOL + ref.HALF_ULP[dtype]) * np.abs(want) + 1e-30 * np.abs(gd * ud)
        ref.close(ref.host(h), want, tol, "h")
        assert ref.guards_intact(h, hbuf)

        dg, gbuf = ref.device_matrix(np.zeros((rows, width)), dtype, pad, offset)
        du, ubuf = ref.device_matrix(np.zeros((rows, width)), dtype, pad, offset)
        _, _, h8 = rip.rip_gate_backward(d, g8, u8, dg, du, hidden=True)
        gk, uk = ref.unpack(*packed(g8), width), ref.unpack(*packed(u8), width)
        dd, s = ref.host(d), ref.sigmoid(gk)
        want = dd * uk * s * (1 + gk * (1 - s))
        mag = np.abs(dd * uk) * (s * (1 + np.abs(gk) * (1 - s)) + 1e-30 * (1 + np.abs(gk)))
        ref.close(ref.host(dg), want, GATE_TOL * mag + ref.HALF_ULP[dtype] * np.abs(want), "dgate")
        want = dd * gk * s
        tol = (GATE_TOL + ref.HALF_ULP[dtype]) * np.abs(want) + 1e-30 * np.abs(dd * gk)
        ref.close(ref.host(du), want, tol, "dup")
        assert ref.guards_intact(dg, gbuf) and ref.guards_intact(du, ubuf)
        # the recomputed product: within half a step of its block, and fp32's error
        hk = ref.unpack(*packed(h8), width)
        want = gk * s * uk
        step = np.repeat(2.0 ** (packed(h8)[1].astype(np.float64) - 127), 32, axis=1)[:, :width]
        ref.close(hk, want, 0.5 * step + GATE_TOL * np.abs(want) + 1e-30, "hidden")
        plain = rip.rip_gate_backward(d, g8, u8)
        assert len(plain) == 2 and torch.equal(plain[0], dg) and torch.equal(plain[1], du)


def test_gate_of_one_projection_side_by_side_and_in_place():
    import torch
    import paper_1909_08029_amd as rip
    torch.manual_seed(5)
    for dtype in (F32, BF16):
        both = torch.randn(33, 2 * 70, device="cuda").to(dtype)
        gate, up = both[:, :70], both[:, 70:]
        h, g8, u8 = rip.rip_gate_forward(gate, up)
        want, _, _ = rip.rip_gate_forward(gate.contiguous(), up.contiguous())
        assert torch.equal(h, want)
        d = torch.randn(33, 70, device="cuda").to(dtype)
        a, b = rip.rip_gate_backward(d, g8, u8)
        dboth = torch.empty_like(both)
        rip.rip_gate_backward(d, g8, u8, dboth[:, :70], dboth[:, 70:])
        assert torch.equal(dboth, torch.cat([a, b], 1))
        own = d.clone()
        a2, b2 = rip.rip_gate_backward(own, g8, u8, dup=own)
        assert b2 is own and torch.equal(a2, a) and torch.equal(own, b)
        copy = gate.contiguous()
        rip.rip_gate_forward(copy, up, out=copy)
        assert torch.equal(copy, want)


def test_gate_gradient_by_differences():
    """At a point that the checkpoints hold exactly, <dh, h> changes along a
    direction as the backward pass says: central differences with step 2^-7 have a
    truncation error of its square times the third derivative (below one here)."""
    import torch
    import paper_1909_08029_amd as rip
    torch.manual_seed(6)
    rows, width, e = 20, 96, 2.0 ** -7
    point = [rip.rip_ckpt_unpack(rip.rip_ckpt_pack(torch.randn(rows, width, device="cuda")), F32)
             for _ in range(2)]
    dh = torch.randn(rows, width, device="cuda")
    _, g8, u8 = rip.rip_gate_forward(*point)
    grads = rip.rip_gate_backward(dh, g8, u8)
    for i in range(2):
        d = torch.randn(rows, width, device="cuda")
        moved = []
        for sign in (1, -1):
            p = list(point)
            p[i] = p[i] + sign * e * d
            moved.append((dh.double() * rip.rip_gate_forward(*p)[0].double()).sum())
        quotient = float(moved[0] - moved[1]) / (2 * e)
        exact = float((grads[i].double() * d.double()).sum())
        size = float((dh.abs() * d.abs() * (1 + point[1 - i].abs())).double().sum())
        assert abs(quotient - exact) <= (e * e + 2.0 ** -16) * size


WGRAD = [  # tokens, out, in, pad, offset
    (1, 1, 1, 0, 0), (0, 5, 40, 0, 0), (1, 40, 33, 0, 0), (7, 129, 70, 1, 3), (31, 16, 32, 0, 0),
    (33, 128, 128, 0, 0), (64, 257, 300, 0, 1), (257, 383, 1000, 0, 0), (1000, 130, 96, 5, 0),
    (5000, 17, 31, 0, 0), (4097, 256, 320, 0, 0), (700, 520, 264, 8, 0)]


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("case", WGRAD, ids=str)
def test_wgrad(case, accumulate):
    import torch
    import paper_1909_08029_amd as rip
    rows, n, k, pad, offset = case
    print(f"case wgrad {case} accumulate={accumulate}", flush=True)
    rng = np.random.default_rng(rows + n * 3 + k)
    x = torch.from_numpy(rng.standard_normal((rows, k)) * 2.0 ** rng.integers(-6, 7, (rows, 1)))
    ck = rip.rip_ckpt_pack(x.float().cuda())
    xk = ref.host(rip.rip_ckpt_unpack(ck, F32))
    for td in (F32, BF16):
        for tg in (F32, BF16):
            dy, _ = ref.device_matrix(rng.standard_normal((rows, n)) * 1e-3, td, pad, offset)
            grad, buf = ref.device_matrix(rng.standard_normal((n, k)), tg, pad, offset)
            start = ref.host(grad) if accumulate else np.zeros((n, k))
            rip.rip_ckpt_wgrad(dy, ck, grad, accumulate=accumulate)
            d = ref.host(dy)
            want = d.T @ xk + start
            mag = np.abs(d).T @ np.abs(xk) + np.abs(start)
            tol = 2 * (rows + 8) * 2.0 ** -24 * mag + ref.HALF_ULP[tg] * np.abs(want)
            ref.close(ref.host(grad), want, tol, f"{td} -> {tg}")
            assert ref.guards_intact(grad, buf)
            if not accumulate:
                again = torch.full_like(grad, 7.0)
                rip.rip_ckpt_wgrad(dy, ck, again)
                assert torch.equal(again, grad)


def test_wgrad_of_fp32_keeps_fp32_accuracy():
    """One token: the gradient is the product dy * x' itself, so all 24 bits of dy
    have to come through the bf16 instructions (three exact parts; the sum of
    their products rounds at most twice)."""
    import torch
    import paper_1909_08029_amd as rip
    rng = np.random.default_rng(9)
    dy = torch.from_numpy(rng.standard_normal((1, 200)).astype(np.float32)).cuda()
    ck = rip.rip_ckpt_pack(torch.from_numpy(rng.standard_normal((1, 64)).astype(np.float32)).cuda())
    grad = rip.rip_ckpt_wgrad(dy, ck, torch.empty(200, 64, device="cuda"))
    want = ref.host(dy).T @ ref.host(rip.rip_ckpt_unpack(ck, F32))
    ref.close(ref.host(grad), want, 2.0 ** -23 * np.abs(want), "outer product")


def test_wgrad_with_infinities_and_nans():
    """They reach the rows and columns that they are in, and no others."""
    import torch
    import paper_1909_08029_amd as rip
    x = torch.ones(40, 64, device="cuda")
    x[3, 40] = float("nan")                       # its block: columns 32..63
    ck = rip.rip_ckpt_pack(x)
    for dtype in (F32, BF16):
        dy = torch.ones(40, 6, device="cuda", dtype=dtype)
        dy[5, 2], dy[6, 4] = float("inf"), float("nan")
        grad = rip.rip_ckpt_wgrad(dy, ck, torch.empty(6, 64, device="cuda"))
        assert torch.isnan(grad[:, 32:]).all()
        assert (grad[[0, 1, 3, 5], :32] == 40).all()
        assert (grad[2, :32] == float("inf")).all() and torch.isnan(grad[4, :32]).all()


def test_refusals():
    import torch
    import paper_1909_08029_amd as rip
    x = torch.zeros(4, 64, device="cuda")
    ck = rip.rip_ckpt_pack(x)
    dy, grad = torch.zeros(4, 8, device="cuda"), torch.zeros(8, 64, device="cuda")
    for call in (lambda: rip.rip_ckpt_pack(x[0]),
                 lambda: rip.rip_ckpt_pack(x, out=rip.Ckpt.empty(4, 65)),
                 lambda: rip.Ckpt(ck.codes, ck.exps, 65),
                 lambda: rip.Ckpt(ck.codes.float(), ck.exps, 64),
                 lambda: rip.Ckpt(ck.codes.t().contiguous().t(), ck.exps, 64),
                 lambda: rip.rip_gate_forward(x, x[:, :32]),
                 lambda: rip.rip_gate_forward(x, x.to(BF16)),
                 lambda: rip.rip_gate_backward(x[:3], ck, ck),
                 lambda: rip.rip_ckpt_wgrad(dy[:3], ck, grad),
                 lambda: rip.rip_ckpt_wgrad(dy, ck, grad[:, :32]),
                 lambda: rip.rip_ckpt_unpack(ck, out=x.t())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        rip.rip_ckpt_pack(x.half())
    other = rip.Ckpt.empty(4, 64)
    d1, d2 = torch.zeros(4, 64, device="cuda"), torch.zeros(5, 64, device="cuda")
    raw = torch.zeros(4 * 64 + 16, dtype=torch.int8, device="cuda")
    odd = rip.Ckpt(raw[1:1 + 256].view(4, 64), ck.exps, 64)
    for call, code in (
            (lambda: rip.rip_gate_forward(x, x, gate_ckpt=other, up_ckpt=other), rip.RIP_E_OVERLAP),
            (lambda: rip.rip_gate_backward(x, ck, other, d1, d1), rip.RIP_E_OVERLAP),
            (lambda: rip.rip_gate_backward(d2[:4], ck, other, d2[1:]), rip.RIP_E_OVERLAP),
            (lambda: rip.rip_gate_backward(x, ck, other, hidden=ck), rip.RIP_E_OVERLAP),
            (lambda: rip.rip_ckpt_pack(x, out=odd), rip.RIP_E_ALIGN),
            (lambda: rip.rip_ckpt_wgrad(grad[:4, :8], ck, grad), rip.RIP_E_OVERLAP),
            (lambda: rip.rip_ckpt_pack(x[:1].expand(4, 64)), rip.RIP_E_INVAL)):
        with pytest.raises(rip.RipError) as e:
            call()
        assert e.value.code == code
