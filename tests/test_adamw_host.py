"""AdamW: refusals before any device call, the step's scalars, and the 8-bit second
moment's format (CPU)."""
import ctypes
import math

import numpy as np
import pytest

import adamw_ref as ref
import paper_1909_08029_amd as rip
from paper_1909_08029_amd import _adamw

A, B, C, D, E, G = (0x10_0000_0000 * i for i in range(1, 7))


def create(n=1, sizes=(100,), dtype=0, fmt=1, **ptr):
    S = len(sizes)
    at = dict(param=A, grad=B, m=C, v=D, m_exps=E, v_exps=G)
    at.update(ptr)
    arrays = [None if p is None else (ctypes.c_void_p * max(1, n * S))(*[p + 4096 * i for i in range(n * S)])
              for p in at.values()]
    h = ctypes.c_void_p()
    rc = rip.lib.rip_adamw_state_create(n, S, dtype, (ctypes.c_int64 * S)(*sizes), *arrays[:2], fmt,
                                        *arrays[2:], ctypes.byref(h))
    assert not h.value
    return rc


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), rip.RIP_E_UNSUPPORTED), (dict(fmt=2), rip.RIP_E_UNSUPPORTED),
    (dict(n=0), rip.RIP_E_INVAL), (dict(n=257), rip.RIP_E_UNSUPPORTED),
    (dict(sizes=(5, -1)), rip.RIP_E_INVAL), (dict(sizes=(1 << 36,)), rip.RIP_E_UNSUPPORTED),
    (dict(sizes=(1 << 34, 1 << 34, 1 << 34)), rip.RIP_E_UNSUPPORTED),
    (dict(param=None), rip.RIP_E_INVAL), (dict(grad=None), rip.RIP_E_INVAL),
    (dict(m=None), rip.RIP_E_INVAL), (dict(v=None), rip.RIP_E_INVAL),
    (dict(m_exps=None), rip.RIP_E_INVAL), (dict(v_exps=None), rip.RIP_E_INVAL),
    (dict(param=0), rip.RIP_E_INVAL),
    (dict(param=A + 2), rip.RIP_E_ALIGN), (dict(grad=B + 1, dtype=1), rip.RIP_E_ALIGN),
    (dict(m=C + 8), rip.RIP_E_ALIGN), (dict(v=D + 1), rip.RIP_E_ALIGN),
    (dict(m=C + 2, fmt=0), rip.RIP_E_ALIGN),
])
def test_refused(change, code):
    assert create(**change) == code
    assert rip.lib.rip_last_error()


def test_null_handles():
    cfg = _adamw._cfg(1e-3, (0.9, 0.999), 1e-8, 0.0, 1.0, 0)
    assert rip.lib.rip_adamw_step(None, None, 0, cfg, 1, None, None) == rip.RIP_E_INVAL
    assert rip.lib.rip_adamw_moments(None, 0, A, B, None) == rip.RIP_E_INVAL
    assert rip.lib.rip_adamw_packed(None) == 0
    assert rip.lib.rip_adamw_scalars_at(None, 1, None) == rip.RIP_E_INVAL
    rip.lib.rip_adamw_state_destroy(None)


def test_scalars():
    for step, lr, betas, wd, gs, seed in ((1, 1e-3, (0.9, 0.999), 0.01, 1.0, 0),
                                          (12345, 0.5, (0.0, 0.0), 0.0, 0.25, -1),
                                          (10 ** 9, 3e-4, (0.95, 0.9999), 0.1, 2.0, 1 << 63)):
        s = rip.rip_adamw_scalars(step, lr, betas, 1e-8, wd, gs, seed)
        want = ref.scalars(step, lr, *betas, wd)
        assert [float(x) for x in s[:4]] == [float(x) for x in want] + [gs]
        k = ref.mix(((seed & (2 ** 64 - 1)) + 0x9E3779B97F4A7C15 * (step + 1)) % 2 ** 64)
        assert list(s[4:].numpy().view(np.uint32)) == [k & 0xffffffff, k >> 32]
    for bad in (dict(step=0), dict(lr=math.inf), dict(betas=(1.0, 0.9)), dict(eps=-1.0)):
        with pytest.raises(rip.RipError):
            rip.rip_adamw_scalars(**dict(dict(step=1, lr=1e-3), **bad))


def test_second_moment_codes():
    """Every code's value is encoded as itself whatever the random bits, codes ascend,
    and a value between two becomes one of them with the right frequency."""
    values = ref.value_v(np.arange(256, dtype=np.uint8), np.full(8, 127, np.uint8))
    assert (np.diff(values) > 0).all() and values[255] == 31 << 14
    for low in (0, 0x7fff0000, 0xffff0000):
        x = np.stack([values, np.full(256, 31 << 14, np.float32)], 1).ravel()  # the largest in each block
        codes, exps = ref.encode_v(x, np.full(512, low, np.uint32))
        assert (codes[::2] == np.arange(256)).all() and (exps == 127).all()
    x = np.array([100.0, 31 << 14], np.float32)   # codes at 96, 100, 104: exact
    x[0] = 101.0                                  # a quarter of the way to 104
    up = [ref.encode_v(x, np.full(2, r << 16, np.uint32))[0][0] for r in range(0, 65536, 64)]
    low = ref.encode_v(np.array([100.0, 31 << 14], np.float32), np.zeros(2, np.uint32))[0][0]
    assert set(up) == {low, low + 1} and np.mean(np.array(up) > low) == 0.25
