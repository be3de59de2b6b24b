"""Plain 64-bit forms of the operators that fill gradient buffers, on the CPU, and
helpers that lay test inputs out (strides, offsets, guards around outputs)."""
import numpy as np
import torch

F32, BF16 = torch.float32, torch.bfloat16
HALF_ULP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}   # bf16: 2^-9 of rounding, and room for it to be
                                                # the other side of a tie
GUARD = 12345.0


def rounded(x, dtype):
    """x (float64 numpy) in a storage type, back as float64."""
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).double().numpy()


def device_matrix(x, dtype, pad=0, offset=0):
    """x (2-D numpy) as a device tensor whose rows are `pad` apart and whose first
    element lies `offset` elements into its buffer, with guard values around it.
    Returns (view, whole buffer)."""
    rows, width = x.shape
    buf = torch.full((rows * (width + pad) + offset + 8,), GUARD, dtype=dtype, device="cuda")
    view = buf[offset:offset + rows * (width + pad)].view(rows, width + pad)[:, :width]
    view.copy_(torch.from_numpy(np.ascontiguousarray(x)).to(dtype))
    return view, buf


def guards_intact(view, buf):
    """Nothing but the view's elements has changed in its buffer."""
    b = buf.clone()
    off = (view.data_ptr() - buf.data_ptr()) // buf.element_size()
    ld = view.stride(0) if view.shape[0] > 1 else view.shape[1]
    for r in range(view.shape[0]):
        b[off + r * ld:off + r * ld + view.shape[1]] = GUARD
    return bool((b == GUARD).all())


def host(t):
    return t.double().cpu().numpy()


def close(got, want, tol, what):
    """|got - want| <= tol elementwise; equal infinities and NaNs in the same places."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = (np.isnan(got) & np.isnan(want)) | (got == want)
    with np.errstate(invalid="ignore"):
        bad = ~same & ~(np.abs(got - want) <= tol)
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        t = np.broadcast_to(tol, got.shape)[i]
        raise AssertionError(f"{what}: {int(bad.sum())} of {got.size} off, first at {i}: "
                             f"{got[i]!r} for {want[i]!r}, tolerance {t:.3g}")


# ---------------------------------------------------------------------------
def embed_grad(dout, ids, vocab, scale):
    """(gradient, sum of magnitudes, tokens of each row)."""
    width = dout.shape[1]
    g, mag, n = np.zeros((vocab, width)), np.zeros((vocab, width)), np.zeros(vocab)
    ok = (ids >= 0) & (ids < vocab)
    np.add.at(g, ids[ok], dout[ok])
    np.add.at(mag, ids[ok], np.abs(dout[ok]))
    np.add.at(n, ids[ok], 1)
    return g * scale, mag * abs(scale), n


def pack(x):
    """(codes, exps) of a float32 matrix, from the format's definition."""
    rows, width = x.shape
    blocks = -(-width // 32)
    b = np.zeros((rows, blocks * 32))
    b[:, :width] = x
    b = b.reshape(rows, blocks, 32)
    codes, exps = np.zeros(b.shape, np.int8), np.zeros((rows, blocks), np.uint8)
    for r in range(rows):
        for c in range(blocks):
            v = b[r, c]
            if not np.isfinite(v).all():
                exps[r, c] = 255
                continue
            e, top = -126, np.abs(v).max()
            if top > 127 * 2.0 ** -126:
                e = int(np.floor(np.log2(top / 127))) - 1
                while top > 127 * 2.0 ** e:
                    e += 1
            codes[r, c], exps[r, c] = np.rint(v / 2.0 ** e), e + 127
    return codes.reshape(rows, blocks * 32), exps


def unpack(codes, exps, width):
    step = np.where(exps == 255, np.nan, 2.0 ** (exps.astype(np.float64) - 127))
    return (codes.astype(np.float64) * np.repeat(step, 32, axis=1))[:, :width]


def sigmoid(x):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-x))


def log_softmax_at(x, targets):
    """(logp, counted, softmax) of each row at its target."""
    n, vocab = x.shape
    counted = (targets >= 0) & (targets < vocab)
    counted &= ~np.all(x == -np.inf, axis=1)
    logp, soft = np.zeros(n), np.zeros(x.shape)
    for t in np.flatnonzero(counted):
        with np.errstate(invalid="ignore", over="ignore"):
            top = x[t].max()
            e = np.exp(x[t] - top)
            soft[t] = e / e.sum()
            logp[t] = x[t, targets[t]] - top - np.log(e.sum())
    return logp, counted, soft


def log_sigmoid(z):
    return np.minimum(z, 0) - np.log1p(np.exp(-np.abs(z)))


def logits_grad(coef, counted, soft, targets):
    g = np.zeros(soft.shape)
    for t in np.flatnonzero(counted & (coef != 0)):
        g[t] = -coef[t] * soft[t]
        g[t, targets[t]] += coef[t]
    return g


def pref_loss(x, targets, offsets, ref, beta, smoothing, grad_scale=1.0):
    logp, counted, soft = log_softmax_at(x, targets)
    seq = np.array([logp[a:b].sum() for a, b in zip(offsets, offsets[1:])])
    pairs = len(ref) // 2
    z = beta * ((seq[0::2] - ref[0::2]) - (seq[1::2] - ref[1::2]))
    loss = np.mean(-(1 - smoothing) * log_sigmoid(z) - smoothing * log_sigmoid(-z))
    c = beta / pairs * (smoothing * sigmoid(z) - (1 - smoothing) * sigmoid(-z)) * grad_scale
    coef = np.zeros(len(x))
    inside = np.zeros(len(x), bool)
    for p in range(pairs):
        for q, sign in ((2 * p, 1), (2 * p + 1, -1)):
            coef[offsets[q]:offsets[q + 1]] = sign * c[p]
            inside[offsets[q]:offsets[q + 1]] = True
    counted = counted & inside
    return dict(loss=loss, seq=seq, logp=np.where(counted, logp, 0), coef=coef, soft=soft,
                counted=counted, grad=logits_grad(coef, counted, soft, targets))


def policy_loss(x, targets, old, adv, weight, ref, low, high, kl, grad_scale=1.0):
    logp, counted, soft = log_softmax_at(x, targets)
    with np.errstate(over="ignore"):
        r = np.exp(logp - old)
        bound = np.clip(r, 1 - low, 1 + high) * adv
        flat = r * adv > bound
        each, slope = -np.minimum(r * adv, bound), np.where(flat, 0, -r * adv)
        if kl:
            d = ref - logp
            each, slope = each + kl * (np.exp(d) - d - 1), slope + kl * (1 - np.exp(d))
    each, slope = np.where(counted, each, 0), np.where(counted, slope, 0)
    coef = weight * slope * grad_scale
    return dict(loss=(weight * each).sum(), logp=np.where(counted, logp, 0), coef=coef, soft=soft,
                counted=counted, grad=logits_grad(coef, counted, soft, targets))
