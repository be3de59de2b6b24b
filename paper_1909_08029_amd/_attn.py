"""Attention of packed sequences with an optional relative position bias, and its
backward pass (binding of that section of include/rip.h; argument marshalling only).

Tensors are [tokens, heads, head_dim]; a token's heads lie side by side, tokens may
have any stride (q, k and v may be parts of one projection's rows).  Streams, devices
and autograd: as for the operators that fill gradient buffers.
"""
from __future__ import annotations

import ctypes
import operator
from typing import NamedTuple, Optional, Sequence, Tuple

import torch

from . import LIB_PATH, _check, lib
from ._train_ops import (_CODES, _device, _elsewhere, _empty, _ids, _matrix, _shaped, _stream,
                         _workspace, _wrote)

MAX_INTERVALS = 128


class _Rel(ctypes.Structure):
    _fields_ = [("n_intervals", ctypes.c_int32), ("starts", ctypes.c_void_p),
                ("rows", ctypes.c_void_p)]


class _Attn(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("q_tokens", ctypes.c_int64),
                ("k_tokens", ctypes.c_int64), ("q_offsets", ctypes.c_void_p),
                ("k_offsets", ctypes.c_void_p), ("n_sequences", ctypes.c_int32),
                ("causal", ctypes.c_int32), ("scale", ctypes.c_float), ("bias", ctypes.c_void_p),
                ("bias_dtype", ctypes.c_int32), ("ld_bias", ctypes.c_int64),
                ("buckets", ctypes.c_int32), ("rel", ctypes.c_void_p)]


def _declare():
    p, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    sigs = {
        "rip_attn_forward_workspace": (i64, [p]),
        "rip_attn_forward": (i32, [p, p, i64, p, i64, p, i64, p, i64, p, p, i64, p, i64, p]),
        "rip_attn_backward_workspace": (i64, [p]),
        "rip_attn_backward": (i32, [p, p, i64, p, i64, p, i64, p, i64, p, p, i64, p, i64, p, i64, p,
                                    i64, p, i64, p, i32, i64, i32, p, i64, p]),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(lib, name, None)
        if fn is None:
            raise ImportError(f"{LIB_PATH} (ABI version {lib.rip_abi_version()}) is older than this "
                              f"package: it has no {name}; run __graft_entry__.build()")
        fn.restype, fn.argtypes = res, args


_declare()


class RelBuckets:
    """Which row of a bias table the distance key - query reads: ``rows[0]`` below
    ``starts[0]``, ``rows[b]`` from ``starts[b - 1]`` on (strictly ascending)."""

    def __init__(self, starts: Sequence[int], rows: Sequence[int]):
        if len(rows) != len(starts) + 1:
            raise ValueError(f"{len(starts)} starts make {len(starts) + 1} intervals, not {len(rows)}")
        self.starts, self.rows = tuple(map(operator.index, starts)), tuple(map(operator.index, rows))
        # the library's lists are int32
        if any(not -2 ** 31 <= x < 2 ** 31 for x in self.starts):
            raise ValueError(f"a start beyond 32 bits: {self.starts}")
        if any(not 0 <= x < 2 ** 31 for x in self.rows):
            raise ValueError(f"rows must be 0 .. 2^31 - 1: {self.rows}")
        self._starts = (ctypes.c_int32 * max(1, len(starts)))(*self.starts)
        self._rows = (ctypes.c_int32 * len(rows))(*self.rows)
        self._rel = _Rel(len(rows), ctypes.addressof(self._starts), ctypes.addressof(self._rows))
        self._address = ctypes.addressof(self._rel)

    @classmethod
    def log(cls, buckets: int, max_distance: int, bidirectional: bool = True) -> "RelBuckets":
        """Buckets whose widths grow with distance (Raffel et al. 2020, section 2.1): half
        of a direction's rows take one distance each, the others grow by a constant
        factor up to ``max_distance``, from which on all distances share the last.
        Earlier keys have the first rows; later keys have the other half of the table,
        or with ``bidirectional`` off share row 0 with the query's own position.  The borders
        are those of exact arithmetic."""
        half = buckets // 2 if bidirectional else buckets
        exact = half // 2
        if exact < 1 or max_distance <= exact or (bidirectional and buckets % 2):
            raise ValueError(f"no buckets: {buckets} rows, distances up to {max_distance}")
        steps, edges, n = half - exact, list(range(exact)), exact
        for i in range(steps):  # n >= exact * (max_distance / exact) ** (i / steps)
            while n ** steps < exact ** (steps - i) * max_distance ** i:
                n += 1
            edges.append(n)
        ends = edges[1:] + [None]
        used = [b for b in range(half) if edges[b] != ends[b]]  # the others hold no distance
        first = {b: edges[b] for b in used}
        left = sorted(used, reverse=True)
        starts = [1 - first[b] for b in left[:-1]]
        rows = list(left)
        if bidirectional:
            starts += [first[b] for b in used if b > 0]
            rows += [half + b for b in used if b > 0]
        return cls(starts, rows)


class Kept(NamedTuple):
    """What the backward pass needs besides out: the rows' log-sums [heads, tokens]
    (float32), and for bfloat16 the rounding errors of out."""
    lse: torch.Tensor
    low: Optional[torch.Tensor]


def _heads(t, name: str, dev: int):
    """(pointer, type, tokens, heads, head_dim, row stride) of [tokens, heads, dim]."""
    if t.get_device() != dev:
        _elsewhere(t, name)
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: unsupported dtype {t.dtype}")
    if t.dim() != 3:
        raise ValueError(f"{name} must be [tokens, heads, head_dim]")
    tokens, heads, dim = t.shape
    ld, across, dense = t.stride()
    if tokens and ((dense != 1 and dim > 1) or (across != dim and heads > 1)):
        raise ValueError(f"{name}: the heads of a token must lie side by side")
    return t.data_ptr(), code, tokens, heads, dim, ld if tokens > 1 else heads * dim


def _like(t, want, name: str, dev: int):
    """(pointer, row stride) of a tensor of the shape and type of `want`."""
    if t.shape != want.shape or t.dtype != want.dtype:
        raise ValueError(f"{name} must be {tuple(want.shape)} of {want.dtype}, not "
                         f"{tuple(t.shape)} of {t.dtype}")
    p, _, _, _, _, ld = _heads(t, name, dev)
    return p, ld


def _problem(q, k, v, q_offsets, k_offsets, causal, scale, bias, buckets, dev):
    """(struct, [(pointer, row stride) of q, k, v])."""
    qp, code, q_tokens, heads, dim, ld_q = _heads(q, "q", dev)
    kp, k_code, k_tokens, kv_heads, k_dim, ld_k = _heads(k, "k", dev)
    vp, ld_v = _like(v, k, "v", dev)
    if code != k_code or dim != k_dim:
        raise ValueError("q, k and v must have one dtype and head_dim")
    op, oc, n = _ids(q_offsets, "q_offsets", dev)
    if oc != 0 or n < 1:
        raise ValueError("q_offsets must hold sequences + 1 int32 values")
    ko = None
    if k_offsets is not None:
        ko, kc, m = _ids(k_offsets, "k_offsets", dev)
        if kc != 0 or m != n:
            raise ValueError("k_offsets must hold as many int32 values as q_offsets")
    if scale is None:
        scale = dim ** -0.5 if dim else 1.0
    a = _Attn(code, heads, kv_heads, dim, q_tokens, k_tokens, op, ko, n - 1, causal, scale)
    if (bias is None) != (buckets is None):
        raise ValueError("bias and buckets go together")
    if bias is not None:
        a.bias, a.bias_dtype, a.buckets, width, a.ld_bias = _matrix(bias, "bias", dev)
        if width != heads:
            raise ValueError(f"bias must be [buckets, {heads}]")
        a.rel = buckets._address
    return a, ((qp, ld_q), (kp, ld_k), (vp, ld_v))


def rip_attn_forward(q, k, v, q_offsets, k_offsets=None, causal: bool = True,
                     scale: Optional[float] = None, bias=None, buckets: Optional[RelBuckets] = None,
                     keep: bool = True, out=None, stream=None) -> Tuple[torch.Tensor, Optional[Kept]]:
    """Attention of packed sequences: q [tokens, heads, head_dim], k and v [keys,
    kv_heads, head_dim], sequence s the rows offsets[s] .. offsets[s + 1] - 1 (int32, on
    the device; k_offsets None: the queries').  A sequence's queries are the last of
    its keys; ``scale`` defaults to head_dim ** -0.5; ``bias`` is a table [buckets,
    heads] read by distance.  Returns (out, Kept for the backward pass, or None without
    ``keep``)."""
    dev = _device()
    a, ((qp, ld_q), (kp, ld_k), (vp, ld_v)) = _problem(q, k, v, q_offsets, k_offsets, causal, scale,
                                                       bias, buckets, dev)
    given = out is not None
    if not given:
        out = _empty(q, q.shape, q.dtype, stream)
    op, ld_out = _like(out, q, "out", dev)
    kept, lse, low, ld_low = None, None, None, 0
    if keep:
        kept = Kept(_empty(q, (a.heads, a.q_tokens), torch.float32, stream),
                    _empty(q, q.shape, q.dtype, stream) if q.dtype is torch.bfloat16 else None)
        lse = kept.lse.data_ptr()
        if kept.low is not None:
            low, ld_low = kept.low.data_ptr(), a.heads * a.head_dim
    ref = ctypes.byref(a)
    nbytes = lib.rip_attn_forward_workspace(ref)
    _keep, ws = _workspace(nbytes, q, stream)
    rc = lib.rip_attn_forward(ref, qp, ld_q, kp, ld_k, vp, ld_v, op, ld_out, lse, low, ld_low, ws,
                              nbytes, _stream(stream, dev))
    if rc:
        _check(rc)
    if given:
        _wrote(out)
    return out, kept


def rip_attn_backward(dout, q, k, v, out, kept: Kept, q_offsets, k_offsets=None,
                      causal: bool = True, scale: Optional[float] = None, bias=None,
                      buckets: Optional[RelBuckets] = None, dbias=None, accumulate: bool = False,
                      dq=None, dk=None, dv=None, stream=None
                      ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dq, dk, dv) from the gradient of out and what rip_attn_forward returned for the
    same arguments; the bias's gradient goes into ``dbias`` [buckets, heads] (a
    replica's gradient segment, say), added to it with ``accumulate``."""
    dev = _device()
    a, ((qp, ld_q), (kp, ld_k), (vp, ld_v)) = _problem(q, k, v, q_offsets, k_offsets, causal, scale,
                                                       bias, buckets, dev)
    op, ld_out = _like(out, q, "out", dev)
    dp, ld_dout = _like(dout, q, "dout", dev)
    lse, low, ld_low = kept.lse, None, 0
    if lse.get_device() != dev:
        _elsewhere(lse, "kept.lse")
    if lse.dtype is not torch.float32 or lse.shape != (a.heads, a.q_tokens) or not lse.is_contiguous():
        raise ValueError(f"kept.lse must be contiguous float32 [{a.heads}, {a.q_tokens}]")
    if kept.low is not None:
        low, ld_low = _like(kept.low, q, "kept.low", dev)
    given = [t for t in (dq, dk, dv, dbias) if t is not None]
    dq = _empty(q, q.shape, q.dtype, stream) if dq is None else dq
    dk = _empty(k, k.shape, k.dtype, stream) if dk is None else dk
    dv = _empty(v, v.shape, v.dtype, stream) if dv is None else dv
    (aq, ld_dq), (ak, ld_dk), (av, ld_dv) = (_like(dq, q, "dq", dev), _like(dk, k, "dk", dev),
                                             _like(dv, k, "dv", dev))
    gp, gc, ld_g = None, 0, 0
    if dbias is not None:
        if bias is None:
            raise ValueError("dbias without a bias")
        gp, gc, _, _, ld_g = _matrix(_shaped(dbias, bias.shape, "dbias"), "dbias", dev)
    ref = ctypes.byref(a)
    nbytes = lib.rip_attn_backward_workspace(ref)
    _keep, ws = _workspace(nbytes, q, stream)
    rc = lib.rip_attn_backward(ref, qp, ld_q, kp, ld_k, vp, ld_v, op, ld_out, lse.data_ptr(), low,
                               ld_low, dp, ld_dout, aq, ld_dq, ak, ld_dk, av, ld_dv, gp, gc, ld_g,
                               1 if accumulate else 0, ws, nbytes, _stream(stream, dev))
    if rc:
        _check(rc)
    for t in given:
        _wrote(t)
    return dq, dk, dv
