"""Attention: refusals before any device call (the addresses are never used), workspace
sizes, and the buckets' borders against exact arithmetic (CPU)."""
import ctypes
from fractions import Fraction

import pytest

import paper_1909_08029_amd as rip
from paper_1909_08029_amd import _attn

A, B, C, D, E, F, G, H, I, J, W = (0x10_0000_0000 * i for i in range(1, 12))   # far apart
INVAL, ALIGN, OVERLAP, UNSUP = (rip.RIP_E_INVAL, rip.RIP_E_ALIGN, rip.RIP_E_OVERLAP, rip.RIP_E_UNSUPPORTED)
BIG = 1 << 40


def problem(starts=(-4, 0), rows=(0, 1, 2), rel=True, intervals=None, no_rows=False, no_starts=False, **change):
    """(struct, what it points to)."""
    at = dict(dtype=1, heads=4, kv_heads=2, head_dim=24, q_tokens=100, k_tokens=150, q_offsets=A,
              k_offsets=A + 4096, n_sequences=3, causal=1, scale=0.5, bias=None, bias_dtype=0, ld_bias=4,
              buckets=3)
    at.update(change)
    s = (ctypes.c_int32 * max(1, len(starts)))(*starts)
    r = (ctypes.c_int32 * max(1, len(rows)))(*rows)
    rb = _attn._Rel(len(rows) if intervals is None else intervals, None if no_starts else ctypes.addressof(s),
                    None if no_rows else ctypes.addressof(r))
    a = _attn._Attn(*at.values(), ctypes.addressof(rb) if rel else None)
    return a, (s, r, rb)


FORWARD = dict(q=B, ld_q=96, k=C, ld_k=48, v=D, ld_v=48, out=E, ld_out=96, lse=F, low=G, ld_low=96, ws=W,
               nbytes=BIG, stream=None)
BACKWARD = dict(q=B, ld_q=96, k=C, ld_k=48, v=D, ld_v=48, out=E, ld_out=96, lse=F, low=G, ld_low=96,
                dout=H, ld_dout=96, dq=I, ld_dq=96, dk=J, ld_dk=48, dv=J + (1 << 30), ld_dv=48, dbias=None,
                dbias_dtype=0, ld_dbias=4, accumulate=0, ws=W, nbytes=BIG, stream=None)


def call(backward, change):
    mats = dict(BACKWARD if backward else FORWARD)
    here = {k: v for k, v in change.items() if k in mats}
    a, _keep = problem(**{k: v for k, v in change.items() if k not in mats})
    mats.update(here)
    name = "rip_attn_backward" if backward else "rip_attn_forward"
    rc = getattr(rip.lib, name)(ctypes.byref(a), *mats.values())
    return rc, getattr(rip.lib, name + "_workspace")(ctypes.byref(a))


BIAS = dict(bias=A + 8192)
BOTH = [
    (dict(dtype=2), UNSUP), (dict(dtype=-1), UNSUP),
    (dict(heads=0), INVAL), (dict(kv_heads=0), INVAL), (dict(head_dim=0), INVAL), (dict(kv_heads=3), INVAL),
    (dict(kv_heads=8), INVAL), (dict(q_tokens=-1), INVAL), (dict(k_tokens=-1), INVAL),
    (dict(n_sequences=-1), INVAL), (dict(n_sequences=(1 << 20) + 1), UNSUP),
    (dict(heads=258), UNSUP), (dict(head_dim=257), UNSUP),
    (dict(q_tokens=(1 << 23) + 1), UNSUP), (dict(k_tokens=(1 << 23) + 1), UNSUP),
    (dict(scale=0.0), INVAL), (dict(scale=-1.0), INVAL), (dict(scale=float("nan")), INVAL),
    (dict(scale=float("inf")), INVAL), (dict(scale=3e38), INVAL),
    (dict(k_offsets=None), INVAL), (dict(q_offsets=None), INVAL),
    (dict(q_offsets=A + 2), ALIGN), (dict(k_offsets=A + 4097), ALIGN),
    (dict(BIAS, rel=False), INVAL), (dict(BIAS, intervals=0), INVAL), (dict(BIAS, no_rows=True), INVAL),
    (dict(BIAS, no_starts=True), INVAL), (dict(BIAS, buckets=0), INVAL),
    (dict(BIAS, buckets=(1 << 20) + 1), UNSUP),
    (dict(BIAS, starts=range(128), rows=[0] * 129), UNSUP),
    (dict(BIAS, rows=(0, 3, 1)), INVAL), (dict(BIAS, rows=(0, -1, 1)), INVAL),
    (dict(BIAS, starts=(4, 4)), INVAL), (dict(BIAS, starts=(4, -4)), INVAL),
    (dict(BIAS, starts=(-1024, 1023)), UNSUP),
    (dict(BIAS, starts=((1 << 24) + 1, (1 << 24) + 2)), UNSUP),
    (dict(BIAS, starts=(-2 ** 31, 2 ** 31 - 1)), UNSUP),
    (dict(BIAS, bias_dtype=2), UNSUP), (dict(BIAS, ld_bias=3), INVAL), (dict(bias=A + 8194), ALIGN),
    (dict(q=None), INVAL), (dict(k=None), INVAL), (dict(v=None), INVAL), (dict(out=None), INVAL),
    (dict(ld_q=95), INVAL), (dict(ld_k=47), INVAL), (dict(ld_v=0), INVAL), (dict(ld_out=1), INVAL),
    (dict(ld_low=95), INVAL),
    (dict(q=B + 1), ALIGN), (dict(v=D + 3), ALIGN), (dict(lse=F + 2), ALIGN), (dict(low=G + 1), ALIGN),
    (dict(ld_q=(1 << 24) + 1), UNSUP), (dict(ld_v=1 << 40), UNSUP),
    (dict(ws=None), INVAL), (dict(nbytes=0), INVAL), (dict(ws=W + 8), ALIGN),
    (dict(ws=B), OVERLAP), (dict(ws=A), OVERLAP), (dict(ws=F - 16), OVERLAP),
]
FORWARD_ONLY = [
    (dict(out=B), OVERLAP), (dict(out=C + 64), OVERLAP), (dict(out=D), OVERLAP), (dict(lse=E), OVERLAP),
    (dict(low=E), OVERLAP), (dict(out=A), OVERLAP), (dict(out=A + 4096), OVERLAP),
    (dict(BIAS, lse=A + 8192), OVERLAP),
]
BACKWARD_ONLY = [
    (dict(dout=None), INVAL), (dict(dq=None), INVAL), (dict(dk=None), INVAL), (dict(dv=None), INVAL),
    (dict(lse=None), INVAL), (dict(dbias=A + 16384), INVAL),
    (dict(BIAS, dbias=A + 16384, ld_dbias=3), INVAL), (dict(BIAS, dbias=A + 16384, dbias_dtype=3), UNSUP),
    (dict(BIAS, dbias=A + 16386), ALIGN), (dict(BIAS, dbias=A + 8192), OVERLAP),
    (dict(dq=B), OVERLAP), (dict(dq=H), OVERLAP), (dict(dk=C), OVERLAP), (dict(dv=J), OVERLAP),
    (dict(dq=E + 2), OVERLAP), (dict(dv=F), OVERLAP), (dict(dk=G), OVERLAP), (dict(BIAS, dbias=I), OVERLAP),
    (dict(ld_dq=95), INVAL), (dict(ld_dk=1 << 40), UNSUP),
]


# (a forward pass of these sizes has a workspace for a bias of many distances only)
@pytest.mark.parametrize("backward,change,code",
                         [(b, c, e) for b in (False, True) for c, e in BOTH] +
                         [(False, c, e) for c, e in FORWARD_ONLY] + [(True, c, e) for c, e in BACKWARD_ONLY])
def test_refused(backward, change, code):
    if not backward and "ws" in change or not backward and "nbytes" in change:
        change = dict(BIAS, starts=(-1000, 0, 1000), rows=(0, 1, 2, 0), **change)
    rc, _ = call(backward, change)
    assert rc == code, rip.lib.rip_last_error()
    assert rip.lib.rip_last_error()


def test_null_problem():
    for backward, name in ((False, "rip_attn_forward"), (True, "rip_attn_backward")):
        mats = BACKWARD if backward else FORWARD
        assert getattr(rip.lib, name)(None, *mats.values()) == INVAL
        assert getattr(rip.lib, name + "_workspace")(None) == 0


def test_workspaces():
    """None of a refused call; of others what the parts and tables need, not more than the
    parts of 64 splits."""
    for fn in (rip.lib.rip_attn_forward_workspace, rip.lib.rip_attn_backward_workspace):
        assert fn(ctypes.byref(problem(heads=0)[0])) == 0
        for bias in (None, A + 8192):
            for n, q, k in ((1, 1, 100000), (8, 8, 5000), (1, 4096, 4096), (1 << 20, 1 << 20, 1 << 20)):
                a, _keep = problem(bias=bias, n_sequences=n, q_tokens=q, k_tokens=k)
                need = fn(ctypes.byref(a))
                parts = 4 * 64 * (q * 4 * 26 + 2 * k * 2 * 24)
                tables = 16 * n + 4 * 4 * q + 4 * 4 * 2100 + 70000
                share = 64 * 4 * 4 * 3 * (q // 128 + n + 2) if bias else 0
                assert 0 <= need <= parts + tables + share, (n, q, k, need)


@pytest.mark.parametrize("buckets", [2, 3, 4, 6, 8, 16, 31, 32, 64])
@pytest.mark.parametrize("far", [2, 3, 9, 20, 100, 128, 1000])
@pytest.mark.parametrize("both", [True, False])
def test_buckets(buckets, far, both):
    """Of every distance the row that the definition gives, in exact arithmetic: bucket
    exact + floor(log(n / exact) / log(far / exact) * (half - exact)), at most half - 1."""
    half = buckets // 2 if both else buckets
    exact = half // 2
    if exact < 1 or far <= exact or (both and buckets % 2):
        with pytest.raises(ValueError):
            rip.RelBuckets.log(buckets, far, both)
        return
    b = rip.RelBuckets.log(buckets, far, both)
    assert list(b.starts) == sorted(set(b.starts)) and len(b.rows) == len(b.starts) + 1
    steps = half - exact
    for rel in range(-far - 5, far + 6):
        n = abs(rel) if both else max(0, -rel)
        if n < exact:
            row = n
        else:                        # the largest i with far^i * exact^(steps - i) <= n^steps
            x, ratio = Fraction(n, exact) ** steps, Fraction(far, exact)
            row = exact + max(i for i in range(steps) if ratio ** i <= x)
        if both and rel > 0:
            row += half
        at = sum(rel >= s for s in b.starts)
        assert b.rows[at] == row, (rel, row)


def test_bucket_arguments():
    with pytest.raises(ValueError):
        rip.RelBuckets([0], [0])
    with pytest.raises(ValueError):
        rip.RelBuckets([], [])
    one = rip.RelBuckets([], [0])
    assert one.starts == () and one.rows == (0,)


FAR = 2 ** 32


@pytest.mark.parametrize("starts,rows", [
    ([FAR + 5], [0, 1]), ([2 ** 31], [0, 1]), ([-2 ** 31 - 1], [0, 1]), ([0, 2 ** 63 - 1], [0, 1, 2]),
    ([0, FAR], [0, 1, 2]), ([0], [0, FAR]), ([0], [0, 2 ** 31]), ([0], [-1, 0]), ([0], [-FAR, 0]),
])
def test_buckets_beyond_32_bits(starts, rows):
    """Numbers that the library's int32 lists would hold as others."""
    with pytest.raises(ValueError):
        rip.RelBuckets(starts, rows)


@pytest.mark.parametrize("starts,rows", [([1.5], [0, 1]), ([0], [0, 1.0]), (["1"], [0, 1]), ([None], [0, 1])])
def test_buckets_that_are_no_integers(starts, rows):
    with pytest.raises(TypeError):
        rip.RelBuckets(starts, rows)


def test_buckets_hold_what_they_show():
    import numpy as np
    b = rip.RelBuckets(np.array([-2 ** 31, 7]), [np.int64(3), 2 ** 31 - 1, True])
    assert b.starts == (-2 ** 31, 7) == tuple(b._starts) and b.rows == (3, 2 ** 31 - 1, 1) == tuple(b._rows)
