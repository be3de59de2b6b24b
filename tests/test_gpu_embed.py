"""Embedding lookup and its gradient against plain 64-bit forms.

Tolerances.  A lookup is one fp32 product and one rounding, reproduced exactly.
A gradient is a sum of n products in fp32: |error| <= (n + 3) 2^-24 * sum of
magnitudes, and the rounding of the result.
"""
import numpy as np
import pytest

import train_ops_ref as ref
from train_ops_ref import BF16, F32

pytestmark = pytest.mark.gpu

TYPES = [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)]


def ids_of(kind, n, vocab, rng):
    if kind == "zipf":
        return np.minimum(((vocab + 1.0) ** rng.random(n) - 1).astype(np.int64), vocab - 1)
    if kind == "same":
        return np.full(n, vocab // 2, np.int64)
    if kind == "none":
        return np.full(n, -1, np.int64)
    ids = rng.integers(-3, vocab + 3, n)
    if kind == "edges" and n > 2:
        ids[:3] = [2 ** 31 - 1, -2 ** 31, vocab]
    return ids


def device_ids(ids, wide):
    import torch
    return torch.from_numpy(ids.astype(np.int64 if wide else np.int32)).cuda()


@pytest.mark.parametrize("n,vocab,width,pad,offset", [
    (1, 1, 1, 0, 0), (1, 7, 1024, 0, 0), (5, 100, 13, 0, 1), (64, 33, 520, 3, 5),
    (257, 1000, 1031, 0, 0), (4099, 50, 40, 8, 0), (3, 9, 4096, 0, 3)])
@pytest.mark.parametrize("types", TYPES, ids=str)
def test_lookup(n, vocab, width, pad, offset, types):
    import torch
    import paper_1909_08029_amd as rip
    rng = np.random.default_rng(n + width)
    table, _ = ref.device_matrix(rng.standard_normal((vocab, width)), types[0], pad, offset)
    ids = ids_of("edges", n, vocab, rng)
    scale = float(np.float32(np.sqrt(width)))
    out, buf = ref.device_matrix(np.zeros((n, width)), types[1], pad, offset)
    for wide in (True, False):
        got = rip.rip_embed_lookup(table, device_ids(ids, wide), scale, out=out)
        assert got is out
        ok = (ids >= 0) & (ids < vocab)
        want = torch.zeros((n, width), dtype=types[1])
        want[torch.from_numpy(ok)] = (table.cpu().float()[ids[ok]] * scale).to(types[1])
        assert torch.equal(out.cpu(), want)
        assert ref.guards_intact(out, buf)


def test_lookup_makes_its_output():
    import torch
    import paper_1909_08029_amd as rip
    table = torch.randn(11, 6, device="cuda")
    ids = torch.tensor([[1, 2, 3], [10, -1, 0]], device="cuda")
    out = rip.rip_embed_lookup(table, ids, dtype=BF16)
    want = (table[ids.clamp(min=0)] * (ids >= 0)[..., None]).to(BF16)
    assert out.shape == (2, 3, 6) and torch.equal(out, want)
    empty = rip.rip_embed_lookup(table, ids[:0])
    assert empty.shape == (0, 3, 6)
    one = rip.rip_embed_lookup(table, torch.tensor(4, device="cuda"))
    assert one.shape == (6,) and torch.equal(one, table[4])


CASES = [  # tokens, vocab, width, ids, pad, offset
    (1, 1, 1, "any", 0, 0), (1, 50, 1024, "zipf", 0, 0), (2, 3, 7, "same", 0, 1),
    (63, 40, 17, "any", 5, 3), (64, 300, 512, "edges", 0, 0), (65, 300, 513, "zipf", 0, 0),
    (129, 1000, 8, "none", 0, 0), (1000, 5, 100, "any", 1, 0), (4096, 70, 24, "zipf", 0, 0),
    (4097, 257, 33, "zipf", 0, 0), (9000, 3, 40, "same", 0, 0), (12289, 66000, 16, "any", 0, 0),
    (20000, 300, 1030, "zipf", 0, 2), (8192, 70000, 8, "edges", 0, 0),
    (70001, 5000, 9, "zipf", 0, 0), (128, 40, 520, "zipf", 0, 0), (40, 3000, 1100, "edges", 0, 1),
    (128, 3, 2100, "same", 0, 0), (1100003, 60, 8, "zipf", 0, 0)]


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_grad(case, accumulate):
    import torch
    import paper_1909_08029_amd as rip
    n, vocab, width, kind, pad, offset = case
    print(f"case embed_grad {case} accumulate={accumulate}", flush=True)
    rng = np.random.default_rng(n * 7 + width)
    ids = ids_of(kind, n, vocab, rng)
    scale = float(np.float32(1.7))
    for i, (td, tg) in enumerate(TYPES):
        dout, _ = ref.device_matrix(rng.standard_normal((n, width)), td, pad, offset)
        before = rng.standard_normal((vocab, width))
        grad, buf = ref.device_matrix(before, tg, pad, offset)
        start = ref.host(grad) if accumulate else 0.0
        dev = device_ids(ids, i % 2 == 0)
        rip.rip_embed_grad(dout, dev, grad, scale, accumulate=accumulate)
        want, mag, cnt = ref.embed_grad(ref.host(dout), ids, vocab, scale)
        want = want + start
        tol = (cnt[:, None] + 3) * 2.0 ** -24 * (mag + np.abs(start)) + ref.HALF_ULP[tg] * np.abs(want)
        ref.close(ref.host(grad), want, tol, f"{td} -> {tg}")
        assert ref.guards_intact(grad, buf)
        if not accumulate:  # the same bits every time
            again = torch.full_like(grad, 7.0)
            rip.rip_embed_grad(dout, dev, again, scale)
            assert torch.equal(again, grad)


def test_grad_is_the_adjoint_of_the_lookup():
    """<dout, lookup(D)> = <grad, D> for every D, as the lookup is linear in its
    table: the difference quotient in every direction is exact."""
    import torch
    import paper_1909_08029_amd as rip
    torch.manual_seed(3)
    ids = torch.randint(-1, 40, (700,), device="cuda")
    dout = torch.randn(700, 96, device="cuda")
    d = torch.randn(40, 96, device="cuda")
    grad = rip.rip_embed_grad(dout, ids, torch.empty_like(d), 0.5)
    lhs = (dout.double() * rip.rip_embed_lookup(d, ids, 0.5).double()).sum()
    rhs = (grad.double() * d.double()).sum()
    assert abs(lhs - rhs) <= 700 * 2.0 ** -24 * float((dout.abs().sum() * d.abs().max()).double())


def test_infinities_and_nans_stay_in_their_rows():
    import torch
    import paper_1909_08029_amd as rip
    ids = torch.tensor([1, 1, 2, -1, 3], device="cuda")
    dout = torch.ones(5, 16, device="cuda")
    dout[0, 3], dout[1, 4], dout[3], dout[2, 0] = float("inf"), float("nan"), float("nan"), 2.0
    grad = rip.rip_embed_grad(dout, ids, torch.full((5, 16), 9.0, device="cuda"))
    assert grad[1, 3] == float("inf") and torch.isnan(grad[1, 4])
    assert torch.isfinite(grad[[0, 2, 3, 4]]).all() and (grad[[0, 4]] == 0).all()
    assert grad[2, 0] == 2 and grad[1, 0] == 2


def test_no_tokens():
    import torch
    import paper_1909_08029_amd as rip
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    dout = torch.empty(0, 20, device="cuda")
    grad = torch.full((6, 20), 3.0, device="cuda")
    rip.rip_embed_grad(dout, ids, grad, accumulate=True)
    assert (grad == 3).all()
    rip.rip_embed_grad(dout, ids, grad)
    assert (grad == 0).all()


def test_offsets_beyond_32_bits():
    """A table and its gradient of more than 2^32 elements."""
    import torch
    import paper_1909_08029_amd as rip
    vocab, width = (1 << 21) + 3, 2053
    table = torch.empty((vocab, width), dtype=BF16, device="cuda")
    table[-1] = torch.arange(width, device="cuda")
    table[0] = 1.0
    ids = torch.tensor([vocab - 1, 0, vocab - 1], device="cuda")
    out = rip.rip_embed_lookup(table, ids)
    assert torch.equal(out, table[ids])
    rip.rip_embed_grad(out, ids, table)
    assert torch.equal(table[-1], out[0] * 2) and (table[0] == 1).all()
    assert (table[1:5] == 0).all() and (table[vocab // 2] == 0).all() and (table[-2] == 0).all()


def test_refusals():
    import torch
    import paper_1909_08029_amd as rip
    table = torch.zeros(10, 16, device="cuda")
    ids = torch.zeros(4, dtype=torch.int64, device="cuda")
    dout = torch.zeros(4, 16, device="cuda")
    for call in (lambda: rip.rip_embed_lookup(table.double(), ids),
                 lambda: rip.rip_embed_lookup(table, ids.float())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: rip.rip_embed_lookup(table.cpu(), ids),
                 lambda: rip.rip_embed_lookup(table, ids.cpu()),
                 lambda: rip.rip_embed_lookup(table.t(), ids),
                 lambda: rip.rip_embed_lookup(table, torch.zeros(8, dtype=torch.int64, device="cuda")[::2]),
                 lambda: rip.rip_embed_lookup(table, ids, out=torch.zeros(4, 15, device="cuda")),
                 lambda: rip.rip_embed_grad(dout[:3], ids, table),
                 lambda: rip.rip_embed_grad(dout[:, :8], ids, table)):
        with pytest.raises(ValueError):
            call()
    for call, code in ((lambda: rip.rip_embed_lookup(table, ids, out=table[2:6]), rip.RIP_E_OVERLAP),
                       (lambda: rip.rip_embed_grad(table[:4], ids, table), rip.RIP_E_OVERLAP),
                       (lambda: rip.rip_embed_grad(dout[:1].expand(4, 16), ids, table), rip.RIP_E_INVAL)):
        with pytest.raises(rip.RipError) as e:
            call()
        assert e.value.code == code
    assert (table == 0).all()
