"""Operators that fill a language-model replica's gradient buffers (binding of
the last section of include/rip.h; argument marshalling only).

Matrices are torch tensors on the current device whose last dimension is dense;
rows may have any stride (a view of a wider buffer).  Tensors of more than two
dimensions are taken as rows of their last one.  Work is enqueued on `stream`
(default: torch's current stream).  Tensors that a call makes, its workspace
among them, are allocated for that stream; the caller makes sure that the inputs
are ready there and keeps them until the stream has passed the call, as with any
tensor used on a second stream.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from . import RIP_BF16, RIP_FP32, _check, _stream_ptr, lib

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
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args


_declare()


def _here(t, name: str):
    if not t.is_cuda or t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{name} must be on the current CUDA device, not {t.device}")


def _matrix(t, name: str):
    """(pointer, type, rows, width, row stride) of a tensor taken as rows."""
    _here(t, name)
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: unsupported dtype {t.dtype}")
    if t.dim() != 2:
        if t.dim() < 2:
            raise ValueError(f"{name} must have at least two dimensions")
        t = t.view(-1, t.shape[-1])
    rows, width = t.shape
    if rows and width > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: the last dimension must be dense")
    return t.data_ptr(), code, rows, width, t.stride(0) if rows > 1 else width


def _ids(t, name: str):
    """(pointer, type, count) of a dense tensor of ids."""
    _here(t, name)
    code = _IDS.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: ids are int32 or int64, not {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr(), code, t.numel()


def _floats(t, name: str, n: int):
    """Pointer of n dense fp32 values; None passes."""
    if t is None:
        return None
    _here(t, name)
    if t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must hold {n} contiguous float32 values")
    return t.data_ptr()


def _empty(shape, dtype, stream):
    """A tensor of the pool of the stream that uses it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device="cuda")
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device="cuda")


def _workspace(nbytes: int, stream):
    """(tensor that keeps it, address) of a call's workspace."""
    if nbytes == 0:
        return None, None
    t = _empty((nbytes,), torch.uint8, stream)
    return t, t.data_ptr()


def _out(given, shape, dtype, name: str, stream):
    if given is None:
        return _empty(shape, dtype, stream)
    if tuple(given.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(given.shape)}")
    return given


# ---------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------
def rip_embed_lookup(table, ids, scale: float = 1.0, dtype=None, out=None, stream=None):
    """scale * table[ids], of ``dtype`` (default: the table's); rows of zeros for
    ids outside the table.  Returns a tensor of shape ids.shape + (width,)."""
    tp, tc, vocab, width, ld = _matrix(table, "table")
    ip, ic, n = _ids(ids, "ids")
    out = _out(out, (*ids.shape, width), dtype or table.dtype, "out", stream)
    op, oc, _, _, ld_out = _matrix(out if out.dim() > 1 else out.view(1, -1), "out")
    _check(lib.rip_embed_lookup(tp, tc, vocab, width, ld, ip, ic, n, scale, op, oc, ld_out,
                                _stream_ptr(stream)))
    return out


def rip_embed_grad(dout, ids, grad, scale: float = 1.0, accumulate: bool = False, stream=None):
    """Gradient of rip_embed_lookup's table into ``grad`` (a replica's gradient
    segment, say): every row is written, or with ``accumulate`` the rows of the
    ids are added to.  Returns grad."""
    dp, dc, rows, width, ld = _matrix(dout if dout.dim() > 1 else dout.view(1, -1), "dout")
    ip, ic, n = _ids(ids, "ids")
    gp, gc, vocab, width_g, ld_g = _matrix(grad, "grad")
    if rows != n or width != width_g:
        raise ValueError(f"dout is {rows} x {width} for {n} ids and a table of width {width_g}")
    nbytes = lib.rip_embed_grad_workspace(n, width)
    _keep, ws = _workspace(nbytes, stream)
    _check(lib.rip_embed_grad(dp, dc, ld, ip, ic, n, scale, gp, gc, vocab, width, ld_g,
                              int(accumulate), ws, nbytes, _stream_ptr(stream)))
    return grad


# ---------------------------------------------------------------------------
# activations in 8 bits
# ---------------------------------------------------------------------------
class Ckpt:
    """A matrix of activations kept in 8 bits (format: include/rip.h): ``codes``
    int8 [rows, 32 * blocks], ``exps`` uint8 [rows, blocks], blocks =
    ceil(width / 32)."""

    __slots__ = ("codes", "exps", "rows", "width")

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
        self.codes, self.exps, self.rows, self.width = codes, exps, rows, width

    @classmethod
    def empty(cls, rows: int, width: int, stream=None) -> "Ckpt":
        blocks = -(-width // BLOCK)
        return cls(_empty((rows, blocks * BLOCK), torch.int8, stream),
                   _empty((rows, blocks), torch.uint8, stream), width)

    def _ptrs(self, name: str):
        _here(self.codes, name)
        _here(self.exps, name)
        return self.codes.data_ptr(), self.exps.data_ptr()


def _ckpt_out(given: Optional[Ckpt], rows: int, width: int, name: str, stream) -> Ckpt:
    if given is None:
        return Ckpt.empty(rows, width, stream)
    if (given.rows, given.width) != (rows, width):
        raise ValueError(f"{name} must be a checkpoint of {rows} x {width}")
    return given


def rip_ckpt_pack(x, out: Optional[Ckpt] = None, stream=None) -> Ckpt:
    """x kept in 8 bits."""
    xp, xc, rows, width, ld = _matrix(x, "x")
    out = _ckpt_out(out, rows, width, "out", stream)
    _check(lib.rip_ckpt_pack(xp, xc, ld, rows, width, *out._ptrs("out"), _stream_ptr(stream)))
    return out


def rip_ckpt_unpack(ckpt: Ckpt, dtype=torch.bfloat16, out=None, stream=None):
    """The values that a checkpoint stands for."""
    out = _out(out, (ckpt.rows, ckpt.width), dtype, "out", stream)
    xp, xc, rows, width, ld = _matrix(out, "out")
    _check(lib.rip_ckpt_unpack(*ckpt._ptrs("ckpt"), rows, width, xp, xc, ld, _stream_ptr(stream)))
    return out


def rip_gate_forward(gate, up, out=None, gate_ckpt: Optional[Ckpt] = None,
                     up_ckpt: Optional[Ckpt] = None, stream=None):
    """(silu(gate) * up, checkpoint of gate, checkpoint of up)."""
    gp, gc, rows, width, ld_g = _matrix(gate, "gate")
    up_, uc, rows_u, width_u, ld_u = _matrix(up, "up")
    out = _out(out, gate.shape, gate.dtype, "out", stream)
    hp, hc, _, _, ld_h = _matrix(out, "out")
    if (rows, width, gc, gc) != (rows_u, width_u, uc, hc):
        raise ValueError("gate, up and out must have one shape and dtype")
    g8 = _ckpt_out(gate_ckpt, rows, width, "gate_ckpt", stream)
    u8 = _ckpt_out(up_ckpt, rows, width, "up_ckpt", stream)
    _check(lib.rip_gate_forward(gp, ld_g, up_, ld_u, gc, rows, width, hp, ld_h,
                                *g8._ptrs("gate_ckpt"), *u8._ptrs("up_ckpt"), _stream_ptr(stream)))
    return out, g8, u8


def rip_gate_backward(dh, gate_ckpt: Ckpt, up_ckpt: Ckpt, dgate=None, dup=None, hidden=False,
                      stream=None):
    """(dgate, dup) from the checkpoints, and with ``hidden`` (True, or a Ckpt to
    fill) also a checkpoint of silu(gate) * up as the third value."""
    dp, dc, rows, width, ld = _matrix(dh, "dh")
    for c in (gate_ckpt, up_ckpt):
        if (c.rows, c.width) != (rows, width):
            raise ValueError(f"dh is {rows} x {width}, a checkpoint is {c.rows} x {c.width}")
    dgate = _out(dgate, dh.shape, dh.dtype, "dgate", stream)
    dup = _out(dup, dh.shape, dh.dtype, "dup", stream)
    ap, ac, _, _, ld_a = _matrix(dgate, "dgate")
    bp, bc, _, _, ld_b = _matrix(dup, "dup")
    if (ac, bc) != (dc, dc):
        raise ValueError("dh, dgate and dup must have one dtype")
    h8 = None
    if hidden is not False and hidden is not None:
        h8 = _ckpt_out(None if hidden is True else hidden, rows, width, "hidden", stream)
    _check(lib.rip_gate_backward(dp, ld, dc, *gate_ckpt._ptrs("gate_ckpt"),
                                 *up_ckpt._ptrs("up_ckpt"), rows, width, ap, ld_a, bp, ld_b,
                                 *((None, None) if h8 is None else h8._ptrs("hidden")),
                                 _stream_ptr(stream)))
    return (dgate, dup) if h8 is None else (dgate, dup, h8)


def rip_ckpt_wgrad(dy, ckpt: Ckpt, grad, accumulate: bool = False, stream=None):
    """dy^T x from the checkpoint of x, into ``grad`` [out_features, in_features]
    (added to it with ``accumulate``).  Returns grad."""
    dp, dc, rows, n, ld = _matrix(dy, "dy")
    gp, gc, n_g, k, ld_g = _matrix(grad, "grad")
    if (rows, n, k) != (ckpt.rows, n_g, ckpt.width):
        raise ValueError(f"dy {rows} x {n}, checkpoint {ckpt.rows} x {ckpt.width} and grad "
                         f"{n_g} x {k} do not fit")
    nbytes = lib.rip_ckpt_wgrad_workspace(dc, rows, n, k)
    _keep, ws = _workspace(nbytes, stream)
    _check(lib.rip_ckpt_wgrad(dp, dc, ld, rows, n, *ckpt._ptrs("ckpt"), k, gp, gc, ld_g,
                              int(accumulate), ws, nbytes, _stream_ptr(stream)))
    return grad


# ---------------------------------------------------------------------------
# losses over the vocabulary
# ---------------------------------------------------------------------------
def _loss_args(logits, targets, grad):
    lp, lc, n, vocab, ld = _matrix(logits, "logits")
    tp, tc, m = _ids(targets, "targets")
    if m != n:
        raise ValueError(f"{n} rows of logits for {m} targets")
    gp, ld_g = None, 0
    if grad is not None:
        gp, gc, n_g, v_g, ld_g = _matrix(grad, "grad")
        if (gc, n_g, v_g) != (lc, n, vocab):
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
    lp, lc, ld, n, vocab, tp, tc, gp, ld_g = _loss_args(logits, targets, grad)
    op, oc, m = _ids(seq_offsets, "seq_offsets")
    if oc != 0 or m < 3 or m % 2 == 0:
        raise ValueError("seq_offsets must hold 2 * pairs + 1 int32 values")
    pairs = m // 2
    rp = _floats(ref_logp, "ref_logp", 2 * pairs)
    out = _empty((1 + 2 * pairs + n,), torch.float32, stream)
    base = out.data_ptr()
    nbytes = lib.rip_pref_loss_workspace(n, vocab, pairs)
    _keep, ws = _workspace(nbytes, stream)
    _check(lib.rip_pref_loss(lp, lc, ld, n, vocab, tp, tc, op, pairs, rp, beta, smoothing,
                             grad_scale, base, base + 4, base + 4 + 8 * pairs, gp, ld_g, ws,
                             nbytes, _stream_ptr(stream)))
    return out[0], out[1:1 + 2 * pairs], out[1 + 2 * pairs:]


def rip_policy_loss(logits, targets, old_logp, advantage, weight=None, ref_logp=None,
                    clip_low: float = 0.2, clip_high: float = 0.2, kl: float = 0.0, grad=None,
                    grad_scale: float = 1.0, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Clipped policy loss with a KL term against ``ref_logp`` (see include/rip.h);
    ``grad`` as in rip_pref_loss.  Returns (loss, log-probabilities of the
    tokens)."""
    lp, lc, ld, n, vocab, tp, tc, gp, ld_g = _loss_args(logits, targets, grad)
    if old_logp is None or advantage is None:
        raise ValueError("old_logp and advantage are needed")
    old, adv = _floats(old_logp, "old_logp", n), _floats(advantage, "advantage", n)
    w, ref = _floats(weight, "weight", n), _floats(ref_logp, "ref_logp", n)
    out = _empty((1 + n,), torch.float32, stream)
    base = out.data_ptr()
    nbytes = lib.rip_policy_loss_workspace(n, vocab)
    _keep, ws = _workspace(nbytes, stream)
    _check(lib.rip_policy_loss(lp, lc, ld, n, vocab, tp, tc, old, adv, w, ref, clip_low, clip_high,
                               kl, grad_scale, base, base + 4, gp, ld_g, ws, nbytes,
                               _stream_ptr(stream)))
    return out[0], out[1:]
