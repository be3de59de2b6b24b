"""The gradient operators at sizes that take the code of large calls: four rows of a
lookup to a thread, gradients wider than a workgroup's columns, rows of logits that
pass a workgroup's registers, every number of threads to a row, and inputs past the
caches.  (The weight gradient's tiles: test_gpu_wgrad_tiles.py.)  The losses and
the embedding run the checks of test_gpu_losses.py and test_gpu_embed.py."""
import pytest

import test_gpu_embed as embed
import test_gpu_losses as losses
import train_ops_ref as ref
from train_ops_ref import BF16, F32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("types", embed.TYPES, ids=str)
@pytest.mark.parametrize("n,vocab,width,pad,offset", [
    (4099, 2000, 1031, 8, 3), (4097, 500, 1024, 0, 0), (65537, 300, 64, 0, 1)])
def test_lookup_of_four_rows_a_thread(n, vocab, width, pad, offset, types):
    assert n * -(-width // 8) >= 1 << 19   # where a thread takes four
    embed.test_lookup(n, vocab, width, pad, offset, types)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("case", [
    (300, 40, 4100, "zipf", 0, 0), (5000, 50, 2500, "edges", 3, 1), (9000, 60, 2055, "zipf", 0, 0)],
    ids=str)
def test_sorted_gradient_wider_than_2048(case, accumulate):
    embed.test_grad(case, accumulate)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("shape", [
    # a whole row to a workgroup; rows in ten and two parts
    (1030, 8209, 0, 0, True), (1030, 17003, 1, 3, False), (200, 100003, 0, 1, True),
    (1000, 32768, 0, 0, True)], ids=str)
def test_pref_loss_of_long_rows(shape, dtype):
    losses.test_pref_loss(shape, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("shape", [
    # 64, 256 and 512 threads to a row, at and beside the limits; more of a row than
    # 512 threads hold; rows split over workgroups
    (70, 2048, 0, 0, True), (70, 2049, 0, 0, True), (40, 5003, 1, 1, False), (70, 16384, 0, 0, True),
    (520, 16385, 7, 0, True), (520, 40009, 1, 3, True), (515, 70016, 0, 0, False),
    (511, 16385, 0, 0, True), (100, 90001, 0, 1, True)], ids=str)
def test_policy_loss_of_every_form(shape, dtype):
    losses.test_policy_loss(shape, dtype)


@pytest.mark.parametrize("dtype,rows,width", [(BF16, 8200, 8209), (BF16, 8200, 8200), (F32, 4100, 8209)],
                         ids=str)
def test_gate_of_inputs_past_the_caches(dtype, rows, width):
    """More than 256 MiB of inputs are read past the caches: the same bits as part by
    part, which is not, and the formulas in 64 bits (tolerances as in
    test_gpu_ckpt.py)."""
    import torch
    import paper_1909_08029_amd as rip
    size = 2 if dtype is BF16 else 4
    assert rows * width * size * 2 > 256 << 20
    gen = torch.Generator(device="cuda").manual_seed(rows + width)
    g, u, d = (torch.randn(rows, width, generator=gen, device="cuda").to(dtype) for _ in range(3))
    h, g8, u8 = rip.rip_gate_forward(g, u)
    dg, du, h8 = rip.rip_gate_backward(d, g8, u8, hidden=True)
    plain = rip.rip_gate_backward(d, g8, u8)
    assert torch.equal(plain[0], dg) and torch.equal(plain[1], du)
    tol, half = 2.0 ** -20, ref.HALF_ULP[dtype]
    for a in range(0, rows, 1025):
        part = slice(a, min(rows, a + 1025))
        ph, pg8, pu8 = rip.rip_gate_forward(g[part], u[part])
        pdg, pdu, ph8 = rip.rip_gate_backward(d[part], pg8, pu8, hidden=True)
        for whole, piece in ((h, ph), (dg, pdg), (du, pdu)):
            assert torch.equal(whole[part], piece)
        for whole, piece in ((g8, pg8), (u8, pu8), (h8, ph8)):
            assert torch.equal(whole.codes[part], piece.codes) and torch.equal(whole.exps[part], piece.exps)
        for given, kept in ((g, pg8), (u, pu8)):
            alone = rip.rip_ckpt_pack(given[part])
            assert torch.equal(alone.codes, kept.codes) and torch.equal(alone.exps, kept.exps)
        gd, ud, dd = g[part].double(), u[part].double(), d[part].double()
        want = gd * torch.sigmoid(gd) * ud
        assert ((ph.double() - want).abs() <= (tol + half) * want.abs() + 1e-30).all()
        gk, uk = rip.rip_ckpt_unpack(pg8, F32).double(), rip.rip_ckpt_unpack(pu8, F32).double()
        s = torch.sigmoid(gk)
        want = dd * uk * s * (1 + gk * (1 - s))
        mag = (dd * uk).abs() * s * (1 + gk.abs() * (1 - s))
        assert ((pdg.double() - want).abs() <= tol * mag + half * want.abs() + 1e-30).all()
        want = dd * gk * s
        assert ((pdu.double() - want).abs() <= (tol + half) * want.abs() + 1e-30).all()
