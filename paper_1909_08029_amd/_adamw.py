"""AdamW as the replicas' local update (binding of that section of include/rip.h;
argument marshalling only)."""
from __future__ import annotations

import ctypes
import operator
import struct
from typing import Optional, Sequence, Tuple

import torch

from . import LIB_PATH, Replicas, _check, _i32_call, lib
from ._train_ops import _CODES, _device, _elsewhere, _empty, _stream, _wrote

STATE_FP32 = 0
STATE_8BIT = 1

BLOCK = 32  # elements that share an exponent


class _Scalars(ctypes.Structure):
    _fields_ = [("decay", ctypes.c_float), ("rate", ctypes.c_float), ("root", ctypes.c_float),
                ("grad_scale", ctypes.c_float), ("key", ctypes.c_uint32 * 2)]


def _declare():
    p, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    sigs = {
        "rip_adamw_state_create": (i32, [i32, i32, i32, p, p, p, i32, p, p, p, p,
                                         ctypes.POINTER(p)]),
        "rip_adamw_state_destroy": (None, [p]),
        "rip_adamw_scalars_at": (i32, [p, i64, p]),
        "rip_adamw_step": (i32, [p, p, i32, p, i64, p, p]),
        "rip_adamw_packed": (i64, [p]),
        "rip_adamw_moments": (i32, [p, i32, p, p, p]),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(lib, name, None)
        if fn is None:
            raise ImportError(f"{LIB_PATH} (ABI version {lib.rip_abi_version()}) is older than this "
                              f"package: it has no {name}; run __graft_entry__.build()")
        fn.restype, fn.argtypes = res, args


_declare()


def _counted(tensors):
    """One tensor for each version counter of these: a view has its base's."""
    bases = [t if t._base is None else t._base for t in tensors]
    return list({id(t): t for t in bases}.values())


class AdamwState:
    """The AdamW moments of the replicas of ``rep`` (which must have gradients).
    ``m[r][s]`` and ``v[r][s]`` hold those of segment s of replica r: contiguous
    float32 tensors of the segment's size, or, with ``m_exps`` and ``v_exps``
    (uint8, one for each block of 32 elements), int8 and uint8 codes in whole
    blocks.  Both formats: include/rip.h.  The tensors must outlive the handle and
    any work enqueued with it."""

    def __init__(self, rep: Replicas, m, v, m_exps=None, v_exps=None):
        param, grad, _ = rep.tensors
        if grad is None:
            raise ValueError("the replicas have no gradient buffers")
        if (m_exps is None) != (v_exps is None):
            raise ValueError("m_exps and v_exps go together")
        self.bits = 32 if m_exps is None else 8
        blocks = [-(-n // BLOCK) for n in rep.numel]
        eight = self.bits == 8
        sizes = [b * BLOCK for b in blocks] if eight else rep.numel
        kinds = [("m", m, torch.int8 if eight else torch.float32, sizes),
                 ("v", v, torch.uint8 if eight else torch.float32, sizes),
                 ("m_exps", m_exps, torch.uint8, blocks), ("v_exps", v_exps, torch.uint8, blocks)]
        for name, rows, dtype, want in kinds:
            if rows is None:
                continue
            if len(rows) != rep.n or any(len(row) != rep.S for row in rows):
                raise ValueError(f"{name} must be N x S tensors")
            for row in rows:
                for t, n in zip(row, want):
                    if t.dtype != dtype or t.numel() != n or not t.is_contiguous() or not t.is_cuda:
                        raise ValueError(f"{name} must hold contiguous CUDA tensors of {dtype} "
                                         f"with {list(want)[:8]} elements")

        def ptrs(rows):
            if rows is None:
                return None
            flat = [t.data_ptr() if t.numel() else None for row in rows for t in row]
            return (ctypes.c_void_p * len(flat))(*flat)

        keep = [ptrs(x) for x in (param, grad, m, v, m_exps, v_exps)]
        self.rep, self.m, self.v, self.m_exps, self.v_exps = rep, m, v, m_exps, v_exps
        h = ctypes.c_void_p()
        _check(lib.rip_adamw_state_create(rep.n, rep.S, rep.dtype, (ctypes.c_int64 * rep.S)(*rep.numel),
                                          *keep[:2], STATE_8BIT if eight else STATE_FP32, *keep[2:],
                                          ctypes.byref(h)))
        self._h = h
        self._destroy = lib.rip_adamw_state_destroy  # still reachable at interpreter exit
        kinds = [rows for rows in (param, m, v, m_exps, v_exps) if rows is not None]
        self._written = [_counted(t for rows in kinds for t in rows[r]) for r in range(rep.n)]
        self._all_written = _counted(t for row in self._written for t in row)

    @classmethod
    def zeros(cls, rep: Replicas, bits: int = 32) -> "AdamwState":
        """New moments of zero, each kind in one buffer for all replicas."""
        if bits not in (32, 8):
            raise ValueError("moments have 32 or 8 bits")
        device = rep.tensors[0][0][0].device

        def make(dtype, unit, size):
            # a segment begins at a whole block, as codes must
            places, at = [], 0
            for n in rep.numel:
                places.append((at, n if size is None else -(-n // BLOCK) * size))
                at += -(-n // BLOCK) * unit
            flat = torch.zeros(rep.n, max(1, at), dtype=dtype, device=device)
            return [[row[a:a + n] for a, n in places] for row in flat]

        if bits == 32:
            return cls(rep, make(torch.float32, BLOCK, None), make(torch.float32, BLOCK, None))
        return cls(rep, make(torch.int8, BLOCK, BLOCK), make(torch.uint8, BLOCK, BLOCK),
                   make(torch.uint8, 1, 1), make(torch.uint8, 1, 1))

    def moments(self, dtype=torch.float32, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
        """(m, v): the values that 8-bit moments stand for, [replicas, elements], a
        replica's segments one after another, each in whole blocks of 32."""
        code = _CODES.get(dtype)
        if code is None:
            raise TypeError(f"unsupported dtype {dtype}")
        shape = (self.rep.n, lib.rip_adamw_packed(self._h))
        like = self.m[0][0]
        m, v = _empty(like, shape, dtype, stream), _empty(like, shape, dtype, stream)
        _check(lib.rip_adamw_moments(self._h, code, m.data_ptr(), v.data_ptr(),
                                     _stream(stream, _device())))
        return m, v

    def close(self):
        if getattr(self, "_h", None):
            self._destroy(self._h)
            self._h = None

    __del__ = close


_PACK = struct.Struct("=6dQ").pack  # of struct rip_adamw: lr .. grad_scale, seed


def _cfg(lr, betas, eps, weight_decay, grad_scale, seed) -> bytes:
    """struct rip_adamw of these values as they are now (a tensor may change in place)."""
    beta1, beta2 = betas
    seed = operator.index(seed) & (2 ** 64 - 1)
    try:
        return _PACK(lr, beta1, beta2, eps, weight_decay, grad_scale, seed)
    except struct.error as e:
        raise TypeError(f"AdamW's settings must be real numbers: {e}") from None


def rip_adamw_scalars(step: int, lr: float, betas: Tuple[float, float] = (0.9, 0.999),
                      eps: float = 1e-8, weight_decay: float = 0.01, grad_scale: float = 1.0,
                      seed: int = 0) -> torch.Tensor:
    """What changes from step to step, as six float32 on the host: decay, rate, root,
    grad_scale and two words of a key.  A copy on the device is rip_adamw_step's
    ``scalars``."""
    out = torch.empty(6, dtype=torch.float32)
    _check(lib.rip_adamw_scalars_at(_cfg(lr, betas, eps, weight_decay, grad_scale, seed), step,
                                    out.data_ptr()))
    return out


def rip_adamw_step(state: AdamwState, active: Sequence[int], step: int, lr: float,
                   betas: Tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
                   weight_decay: float = 0.01, grad_scale: float = 1.0, seed: int = 0,
                   scalars: Optional[torch.Tensor] = None, stream=None) -> None:
    """AdamW step ``step`` (1, 2, ...) of the ``active`` workers in one launch (see
    include/rip.h).  ``scalars`` on the device (rip_adamw_scalars) takes the place
    of what lr, weight_decay, grad_scale, seed and step say, read when the launch
    runs: for graphs replayed with later steps' scalars.  The workers' parameters and
    moments count as modified in place."""
    live = None
    if scalars is not None:
        if scalars.get_device() != _device():
            _elsewhere(scalars, "scalars")
        if scalars.dtype is not torch.float32 or scalars.numel() != 6 or not scalars.is_contiguous():
            raise ValueError("scalars must hold six contiguous float32 values (rip_adamw_scalars)")
        live = scalars.data_ptr()
    act, ids = _i32_call(list(active))
    rc = lib.rip_adamw_step(state._h, act, len(active),
                            _cfg(lr, betas, eps, weight_decay, grad_scale, seed), step, live,
                            _stream(stream, _device()))
    if rc:
        _check(rc)
    if len(active) == state.rep.n:
        _wrote(state._all_written)
    else:
        _wrote([t for r in ids[:len(active)] for t in state._written[r]])
