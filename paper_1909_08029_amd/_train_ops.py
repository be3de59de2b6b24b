"""Operators that fill a language-model replica's gradient buffers (binding of
the last section of include/rip.h; argument marshalling only).

Matrices are torch tensors on the current device whose last dimension is dense;
rows may have any stride (a view of a wider buffer).  Tensors of more than two
dimensions are taken as rows of their last one.  Work is enqueued on `stream`
(default: torch's current stream).  Tensors that a call makes, its workspace
among them, are allocated for that stream; the caller makes sure that the inputs
are ready there and keeps them until the stream has passed the call, as with any
tensor used on a second stream.

The calls stand outside automatic differentiation, as a backward pass written by
hand does: a tensor that requires grad is taken as its values, and nothing that a
call returns requires grad.  A tensor that a call writes counts as modified in
place, so that autograd refuses a later backward pass that would have needed what
it held before (logits under their own gradient, say).
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import LIB_PATH, RIP_BF16, RIP_FP32, _check, _raw_stream, _stream_ptr, lib

_CODES = {torch.float32: RIP_FP32, torch.bfloat16: RIP_BF16}
_IDS = {torch.int32: 0, torch.int64: 1}

BLOCK = 32  # columns of a checkpoint block


def _declare():
    p, i32, i64, f = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    sigs = {
        "rip_embed_lookup": (i32, [p, i32, i64, i64, i64, p, i32, i64, f, p, i32, i64, p]),
        "rip_embed_grad_workspace": (i64, [i64, i64]),
        "rip_embed_grad": (i32, [p, i32, i64, p, i32, i64, f, p, i32, i64, i64, i64, i32, p, i64,
                                 p]),
        "rip_ckpt_pack": (i32, [p, i32, i64, i64, i64, p, p, p]),
        "rip_ckpt_unpack": (i32, [p, p, i64, i64, p, i32, i64, p]),
        "rip_gate_forward": (i32, [p, i64, p, i64, i32, i64, i64, p, i64, p, p, p, p, p]),
        "rip_gate_backward": (i32, [p, i64, i32, p, p, p, p, i64, i64, p, i64, p, i64, p, p, p]),
        "rip_ckpt_wgrad_workspace": (i64, [i32, i64, i64, i64]),
        "rip_ckpt_wgrad": (i32, [p, i32, i64, i64, i64, p, p, i64, p, i32, i64, i32, p, i64, p]),
        "rip_pref_loss_workspace": (i64, [i64, i64, i32]),
        "rip_pref_loss": (i32, [p, i32, i64, i64, i64, p, i32, p, i32, p, f, f, f, p, p, p, p, i64,
                                p, i64, p]),
        "rip_policy_loss_workspace": (i64, [i64, i64]),
        "rip_policy_loss": (i32, [p, i32, i64, i64, i64, p, i32, p, p, p, p, f, f, f, f, p, p, p,
                                  i64, p, i64, p]),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(lib, name, None)
        if fn is None:
            raise ImportError(f"{LIB_PATH} (ABI version {lib.rip_abi_version()}) is older than this "
                              f"package: it has no {name}; run __graft_entry__.build()")
        fn.restype, fn.argtypes = res, args


_declare()


# Marks a caller's tensor as modified in place (0.3 us).
_wrote = torch.autograd.graph.increment_version


# The checks below run on every call of a training loop or a decoding step, so they
# ask each tensor for as little as possible and torch's bookkeeping only once.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _device() -> int:
    """The current device; -2 (no tensor's) while CUDA is not in use."""
    return _current_device() if torch.cuda.is_initialized() else -2


def _stream(stream, dev: int):
    """Raw stream of a call: torch's current one unless given."""
    if stream is None and dev >= 0 and _raw_stream is not None:
        return _raw_stream(dev)
    return _stream_ptr(stream)


def _elsewhere(t, name: str):
    raise ValueError(f"{name} must be on the current CUDA device, not {t.device}")


def _matrix(t, name: str, dev: int):
    """(pointer, type, rows, width, row stride) of a tensor taken as rows."""
    if t.get_device() != dev:
        _elsewhere(t, name)
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: unsupported dtype {t.dtype}")
    shape = t.shape
    if len(shape) != 2:
        if len(shape) < 2:
            raise ValueError(f"{name} must have at least two dimensions")
        t = t.view(-1, shape[-1])
        shape = t.shape
    rows, width = shape
    ld, dense = t.stride()
    if dense != 1 and width > 1 and rows:
        raise ValueError(f"{name}: the last dimension must be dense")
    return t.data_ptr(), code, rows, width, ld if rows > 1 else width


def _ids(t, name: str, dev: int):
    """(pointer, type, count) of a dense tensor of ids."""
    if t.get_device() != dev:
        _elsewhere(t, name)
    code = _IDS.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: ids are int32 or int64, not {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr(), code, t.numel()


def _floats(t, name: str, n: int, dev: int):
    """Pointer of n dense fp32 values; None passes."""
    if t is None:
        return None
    if t.get_device() != dev:
        _elsewhere(t, name)
    if t.dtype is not torch.float32 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must hold {n} contiguous float32 values")
    return t.data_ptr()


def _empty(like, shape, dtype, stream):
    """A tensor on the device of `like`, of the pool of the stream that uses it."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _empty_like(like, stream):
    """A dense tensor of the shape and dtype of `like`."""
    if stream is None:
        return torch.empty_like(like, memory_format=torch.contiguous_format)
    with torch.cuda.stream(stream):
        return torch.empty_like(like, memory_format=torch.contiguous_format)


def _workspace(nbytes: int, like, stream):
    """(tensor that keeps it, address) of a call's workspace."""
    if nbytes == 0:
        return None, None
    t = _empty(like, (nbytes,), torch.uint8, stream)
    return t, t.data_ptr()


def _shaped(given, shape, name: str):
    if given.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(given.shape)}")
    return given


# ---------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------
def rip_embed_lookup(table, ids, scale: float = 1.0, dtype=None, out=None, stream=None):
    """scale * table[ids], of ``dtype`` (default: the table's); rows of zeros for
    ids outside the table.  Returns a tensor of shape ids.shape + (width,)."""
    dev = _device()
    tp, tc, vocab, width, ld = _matrix(table, "table", dev)
    ip, ic, n = _ids(ids, "ids", dev)
    shape = (*ids.shape, width)
    given = out is not None
    if given:
        _shaped(out, shape, "out")
    else:
        out = _empty(table, shape, dtype or table.dtype, stream)
    op, oc, _, _, ld_out = _matrix(out if len(shape) > 1 else out.view(1, -1), "out", dev)
    rc = lib.rip_embed_lookup(tp, tc, vocab, width, ld, ip, ic, n, scale, op, oc, ld_out,
                              _stream(stream, dev))
    if rc:
        _check(rc)
    if given:
        _wrote(out)
    return out


def rip_embed_grad(dout, ids, grad, scale: float = 1.0, accumulate: bool = False, stream=None):
    """Gradient of rip_embed_lookup's table into ``grad`` (a replica's gradient
    segment, say): every row is written, or with ``accumulate`` the rows of the
    ids are added to.  Returns grad."""
    dev = _device()
    dp, dc, rows, width, ld = _matrix(dout if dout.dim() > 1 else dout.view(1, -1), "dout", dev)
    ip, ic, n = _ids(ids, "ids", dev)
    gp, gc, vocab, width_g, ld_g = _matrix(grad, "grad", dev)
    if rows != n or width != width_g:
        raise ValueError(f"dout is {rows} x {width} for {n} ids and a table of width {width_g}")
    nbytes = lib.rip_embed_grad_workspace(n, width)
    _keep, ws = _workspace(nbytes, grad, stream)
    rc = lib.rip_embed_grad(dp, dc, ld, ip, ic, n, scale, gp, gc, vocab, width, ld_g,
                            1 if accumulate else 0, ws, nbytes, _stream(stream, dev))
    if rc:
        _check(rc)
    _wrote(grad)
    return grad


# ---------------------------------------------------------------------------
# activations in 8 bits
# ---------------------------------------------------------------------------
class Ckpt:
    """A matrix of activations kept in 8 bits (format: include/rip.h): ``codes``
    int8 [rows, 32 * blocks], ``exps`` uint8 [rows, blocks], blocks =
    ceil(width / 32).  Made from such tensors, or by the calls below, which keep
    both in one buffer."""

    __slots__ = ("rows", "width", "_codes", "_exps", "_buffer", "_at", "_ptrs", "_dev")

    def __init__(self, codes, exps, width: int):
        blocks = -(-width // BLOCK)
        rows = codes.shape[0]
        if (codes.dtype, exps.dtype) != (torch.int8, torch.uint8) or \
                tuple(codes.shape) != (rows, blocks * BLOCK) or \
                tuple(exps.shape) != (rows, blocks):
            raise ValueError(f"a checkpoint of width {width} has int8 codes [rows, {blocks * BLOCK}] "
                             f"and uint8 exps [rows, {blocks}]")
        if not codes.is_contiguous() or not exps.is_contiguous():
            raise ValueError("codes and exps must be contiguous")
        if codes.device != exps.device:
            raise ValueError("codes and exps must be on one device")
        self.rows, self.width, self._codes, self._exps = rows, width, codes, exps
        self._buffer, self._at = None, None
        self._ptrs, self._dev = (codes.data_ptr(), exps.data_ptr()), codes.get_device()

    @classmethod
    def _make(cls, like, rows: int, width: int, count: int, stream):
        """`count` checkpoints in one buffer: all codes, then all exponents."""
        units = rows * -(-width // BLOCK)
        size = units * BLOCK
        buf = _empty(like, (count * (size + units),), torch.uint8, stream)
        base, dev, out = buf.data_ptr(), buf.get_device(), []
        for i in range(count):
            c = cls.__new__(cls)
            c.rows, c.width, c._codes, c._exps, c._buffer, c._dev = rows, width, None, None, buf, dev
            c._at = (i * size, count * size + i * units)
            c._ptrs = (base + c._at[0], base + c._at[1]) if units else (None, None)
            out.append(c)
        return out

    @classmethod
    def empty(cls, rows: int, width: int, stream=None) -> "Ckpt":
        """One of undefined contents on the current device."""
        like = torch.empty(0, dtype=torch.uint8, device="cuda")
        return cls._make(like, rows, width, 1, stream)[0]

    @property
    def codes(self):
        if self._codes is None:
            blocks = -(-self.width // BLOCK)
            part = self._buffer.narrow(0, self._at[0], self.rows * blocks * BLOCK)
            self._codes = part.view(torch.int8).view(self.rows, blocks * BLOCK)
        return self._codes

    @property
    def exps(self):
        if self._exps is None:
            blocks = -(-self.width // BLOCK)
            part = self._buffer.narrow(0, self._at[1], self.rows * blocks)
            self._exps = part.view(self.rows, blocks)
        return self._exps


def _ckpt(c: Ckpt, rows: int, width: int, name: str, dev: int):
    """Pointers of a checkpoint of these sizes."""
    if c._dev != dev:
        raise ValueError(f"{name} must be on the current CUDA device")
    if c.rows != rows or c.width != width:
        raise ValueError(f"{name} is a checkpoint of {c.rows} x {c.width}, not {rows} x {width}")
    return c._ptrs


def rip_ckpt_pack(x, out: Optional[Ckpt] = None, stream=None) -> Ckpt:
    """x kept in 8 bits."""
    dev = _device()
    xp, xc, rows, width, ld = _matrix(x, "x", dev)
    if out is None:
        out = Ckpt._make(x, rows, width, 1, stream)[0]
    codes, exps = _ckpt(out, rows, width, "out", dev)
    rc = lib.rip_ckpt_pack(xp, xc, ld, rows, width, codes, exps, _stream(stream, dev))
    if rc:
        _check(rc)
    return out


def rip_ckpt_unpack(ckpt: Ckpt, dtype=torch.bfloat16, out=None, stream=None):
    """The values that a checkpoint stands for."""
    dev = _device()
    codes, exps = _ckpt(ckpt, ckpt.rows, ckpt.width, "ckpt", dev)
    shape = (ckpt.rows, ckpt.width)
    given = out is not None
    if given:
        _shaped(out, shape, "out")
    else:
        like = ckpt._codes if ckpt._buffer is None else ckpt._buffer
        out = _empty(like, shape, dtype, stream)
    xp, xc, rows, width, ld = _matrix(out, "out", dev)
    rc = lib.rip_ckpt_unpack(codes, exps, rows, width, xp, xc, ld, _stream(stream, dev))
    if rc:
        _check(rc)
    if given:
        _wrote(out)
    return out


def rip_gate_forward(gate, up, out=None, gate_ckpt: Optional[Ckpt] = None,
                     up_ckpt: Optional[Ckpt] = None, stream=None):
    """(silu(gate) * up, checkpoint of gate, checkpoint of up)."""
    dev = _device()
    gp, gc, rows, width, ld_g = _matrix(gate, "gate", dev)
    up_, uc, rows_u, width_u, ld_u = _matrix(up, "up", dev)
    given = out is not None
    if given:
        hp, hc, _, _, ld_h = _matrix(_shaped(out, gate.shape, "out"), "out", dev)
    else:
        out = _empty_like(gate, stream)
        hp, hc, ld_h = out.data_ptr(), gc, width
    if rows != rows_u or width != width_u or gc != uc or gc != hc:
        raise ValueError("gate, up and out must have one shape and dtype")
    if gate_ckpt is None and up_ckpt is None:
        gate_ckpt, up_ckpt = Ckpt._make(gate, rows, width, 2, stream)
    elif gate_ckpt is None or up_ckpt is None:
        made = Ckpt._make(gate, rows, width, 1, stream)[0]
        gate_ckpt, up_ckpt = gate_ckpt or made, up_ckpt or made
    g_codes, g_exps = _ckpt(gate_ckpt, rows, width, "gate_ckpt", dev)
    u_codes, u_exps = _ckpt(up_ckpt, rows, width, "up_ckpt", dev)
    rc = lib.rip_gate_forward(gp, ld_g, up_, ld_u, gc, rows, width, hp, ld_h, g_codes, g_exps,
                              u_codes, u_exps, _stream(stream, dev))
    if rc:
        _check(rc)
    if given:
        _wrote(out)
    return out, gate_ckpt, up_ckpt


def rip_gate_backward(dh, gate_ckpt: Ckpt, up_ckpt: Ckpt, dgate=None, dup=None, hidden=False,
                      stream=None):
    """(dgate, dup) from the checkpoints, and with ``hidden`` (True, or a Ckpt to
    fill) also a checkpoint of silu(gate) * up as the third value."""
    dev = _device()
    dp, dc, rows, width, ld = _matrix(dh, "dh", dev)
    g_codes, g_exps = _ckpt(gate_ckpt, rows, width, "gate_ckpt", dev)
    u_codes, u_exps = _ckpt(up_ckpt, rows, width, "up_ckpt", dev)
    given = [t for t in (dgate, dup) if t is not None]
    if dgate is None:
        dgate = _empty_like(dh, stream)
        ap, ac, ld_a = dgate.data_ptr(), dc, width
    else:
        ap, ac, _, _, ld_a = _matrix(_shaped(dgate, dh.shape, "dgate"), "dgate", dev)
    if dup is None:
        dup = _empty_like(dh, stream)
        bp, bc, ld_b = dup.data_ptr(), dc, width
    else:
        bp, bc, _, _, ld_b = _matrix(_shaped(dup, dh.shape, "dup"), "dup", dev)
    if ac != dc or bc != dc:
        raise ValueError("dh, dgate and dup must have one dtype")
    h8, h_codes, h_exps = None, None, None
    if hidden is not False and hidden is not None:
        h8 = Ckpt._make(dh, rows, width, 1, stream)[0] if hidden is True else hidden
        h_codes, h_exps = _ckpt(h8, rows, width, "hidden", dev)
    rc = lib.rip_gate_backward(dp, ld, dc, g_codes, g_exps, u_codes, u_exps, rows, width, ap, ld_a,
                               bp, ld_b, h_codes, h_exps, _stream(stream, dev))
    if rc:
        _check(rc)
    for t in given:
        _wrote(t)
    return (dgate, dup) if h8 is None else (dgate, dup, h8)


def rip_ckpt_wgrad(dy, ckpt: Ckpt, grad, accumulate: bool = False, stream=None):
    """dy^T x from the checkpoint of x, into ``grad`` [out_features, in_features]
    (added to it with ``accumulate``).  Returns grad."""
    dev = _device()
    dp, dc, rows, n, ld = _matrix(dy, "dy", dev)
    gp, gc, n_g, k, ld_g = _matrix(grad, "grad", dev)
    if rows != ckpt.rows or n != n_g or k != ckpt.width:
        raise ValueError(f"dy {rows} x {n}, checkpoint {ckpt.rows} x {ckpt.width} and grad "
                         f"{n_g} x {k} do not fit")
    codes, exps = _ckpt(ckpt, rows, k, "ckpt", dev)
    nbytes = lib.rip_ckpt_wgrad_workspace(dc, rows, n, k)
    _keep, ws = _workspace(nbytes, grad, stream)
    rc = lib.rip_ckpt_wgrad(dp, dc, ld, rows, n, codes, exps, k, gp, gc, ld_g,
                            1 if accumulate else 0, ws, nbytes, _stream(stream, dev))
    if rc:
        _check(rc)
    _wrote(grad)
    return grad


# ---------------------------------------------------------------------------
# losses over the vocabulary
# ---------------------------------------------------------------------------
def _loss_args(logits, targets, grad, dev: int):
    lp, lc, n, vocab, ld = _matrix(logits, "logits", dev)
    tp, tc, m = _ids(targets, "targets", dev)
    if m != n:
        raise ValueError(f"{n} rows of logits for {m} targets")
    gp, ld_g = None, 0
    if grad is not None:
        gp, gc, n_g, v_g, ld_g = _matrix(grad, "grad", dev)
        if gc != lc or n_g != n or v_g != vocab:
            raise ValueError("grad must have the logits' shape and dtype")
    return lp, lc, ld, n, vocab, tp, tc, gp, ld_g


def rip_pref_loss(logits, targets, seq_offsets, ref_logp, beta: float = 0.1,
                  smoothing: float = 0.0, grad=None, grad_scale: float = 1.0, stream=None
                  ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Preference loss over pairs of sequences: sequence 2p (chosen) and 2p + 1
    (rejected) of the packed tokens are the rows seq_offsets[q] ..
    seq_offsets[q + 1] - 1 (int32, on the device).  ``grad`` takes grad_scale *
    the gradient of the logits and may be the logits themselves; None computes the
    loss alone.  Returns (loss, log-probabilities of the sequences, of the
    tokens)."""
    dev = _device()
    lp, lc, ld, n, vocab, tp, tc, gp, ld_g = _loss_args(logits, targets, grad, dev)
    op, oc, m = _ids(seq_offsets, "seq_offsets", dev)
    if oc != 0 or m < 3 or m % 2 == 0:
        raise ValueError("seq_offsets must hold 2 * pairs + 1 int32 values")
    pairs = m // 2
    rp = _floats(ref_logp, "ref_logp", 2 * pairs, dev)
    out = _empty(logits, (1 + 2 * pairs + n,), torch.float32, stream)
    base = out.data_ptr()
    nbytes = lib.rip_pref_loss_workspace(n, vocab, pairs)
    _keep, ws = _workspace(nbytes, logits, stream)
    rc = lib.rip_pref_loss(lp, lc, ld, n, vocab, tp, tc, op, pairs, rp, beta, smoothing,
                           grad_scale, base, base + 4, base + 4 + 8 * pairs, gp, ld_g, ws,
                           nbytes, _stream(stream, dev))
    if rc:
        _check(rc)
    if grad is not None:
        _wrote(grad)
    return out[0], out[1:1 + 2 * pairs], out[1 + 2 * pairs:]


def rip_policy_loss(logits, targets, old_logp, advantage, weight=None, ref_logp=None,
                    clip_low: float = 0.2, clip_high: float = 0.2, kl: float = 0.0, grad=None,
                    grad_scale: float = 1.0, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Clipped policy loss with a KL term against ``ref_logp`` (see include/rip.h);
    ``grad`` as in rip_pref_loss.  Returns (loss, log-probabilities of the
    tokens)."""
    dev = _device()
    lp, lc, ld, n, vocab, tp, tc, gp, ld_g = _loss_args(logits, targets, grad, dev)
    if old_logp is None or advantage is None:
        raise ValueError("old_logp and advantage are needed")
    old, adv = _floats(old_logp, "old_logp", n, dev), _floats(advantage, "advantage", n, dev)
    w, ref = _floats(weight, "weight", n, dev), _floats(ref_logp, "ref_logp", n, dev)
    out = _empty(logits, (1 + n,), torch.float32, stream)
    base = out.data_ptr()
    nbytes = lib.rip_policy_loss_workspace(n, vocab)
    _keep, ws = _workspace(nbytes, logits, stream)
    rc = lib.rip_policy_loss(lp, lc, ld, n, vocab, tp, tc, old, adv, w, ref, clip_low, clip_high,
                             kl, grad_scale, base, base + 4, gp, ld_g, ws, nbytes,
                             _stream(stream, dev))
    if rc:
        _check(rc)
    if grad is not None:
        _wrote(grad)
    return out[0], out[1:]
