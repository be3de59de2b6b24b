"""Attention with a relative position bias and its gradients in 64 bits, from the
definition in include/rip.h (torch, any device), with bounds of what the roundings
that the definition allows can do to each element.

Bounds.  u = 2^-24 (fp32), h = half a step of the inputs' type (2^-8 bf16; fp32: u).
  score    |dx| <= X = u (d + 4) scale sum |q||k| + 4 u (|x| + |bias|): d products added
           in any order, scaled, the bias added, all in fp32
  p        relative error g = 2 X' + 8 u (X' the largest X of the row; its own score and
           the row's log-sum; the exponential and the normalisation)
  out, dv  h for p as the product takes it (2^-16 for out where it is taken as two
           numbers), g, and n u for a sum of n terms, all of sum p |v|; the result's
           rounding
  ds       (g + (d + 4) u) p (sum |dout||v| + sum |dout||out|) and what delta has from
           out: out's own error above (its rounding too where low is not there, 2^-16 of
           it where it is), times |dout|
  dq, dk   h |ds| (as the product takes it), the error of ds and n u |ds|, times
           |k| or |q|; the result's rounding
  dbias    the error of ds and n u |ds| over the bucket; the result's rounding
"""
import math

import torch

U = 2.0 ** -24


def cleaned(offsets, total):
    """Offsets as a call takes them: within 0 .. total and no smaller than those before."""
    out, most = [], 0
    for x in offsets:
        most = max(most, min(max(int(x), 0), total))
        out.append(most)
    return out


def interval_rows(rel, starts, rows):
    at = torch.zeros_like(rel)
    for s in starts:
        at += rel >= s
    return torch.tensor(rows, device=rel.device)[at]


class Attention:
    """Results in float64 and, for each, a bound of its elements' errors (`tol`)."""
    NAMES = ("out", "lse", "dq", "dk", "dv", "dbias")

    def __init__(self, q, k, v, q_offsets, k_offsets=None, causal=True, scale=None, bias=None, starts=(),
                 rows=(0,), dout=None, low=True):
        h = 2.0 ** -8 if q.dtype == torch.bfloat16 else U
        exact = h == U or (bias is not None and low)
        p_step = (2.0 ** -16 if exact else h) if h != U else U
        kept = U if h == U else 2.0 ** -16 if low else h      # of out, as delta takes it
        bias_step = 0.0 if bias is None else (2.0 ** -8 if bias.dtype == torch.bfloat16 else U)
        dev = q.device
        q, k, v = (x.detach().double() for x in (q, k, v))
        bias = None if bias is None else bias.detach().double()
        if bias is not None:
            bias = torch.where(bias < -65536, -math.inf, bias)
        heads, group, d = q.shape[1], q.shape[1] // k.shape[1], q.shape[2]
        scale = d ** -0.5 if scale is None else scale
        qo = cleaned(q_offsets, len(q))
        ko = qo if k_offsets is None else cleaned(k_offsets, len(k))
        new = lambda x: torch.zeros_like(x)  # noqa: E731
        self.out, self.dq, self.dk, self.dv = new(q), new(q), new(k), new(v)
        self.lse = torch.full((heads, len(q)), -math.inf, dtype=torch.float64, device=dev)
        self.dbias = None if bias is None else torch.zeros_like(bias)
        tol = {n: torch.zeros_like(getattr(self, n)) for n in self.NAMES
               if getattr(self, n) is not None}
        for a, b, ka, kb in zip(qo, qo[1:], ko, ko[1:]):
            if a == b or ka == kb:
                continue
            n = kb - ka
            pos = torch.arange(b - a, device=dev) + n - (b - a)
            rel = torch.arange(n, device=dev)[None, :] - pos[:, None]
            row = None if bias is None else interval_rows(rel, starts, rows)
            for hd in range(heads):
                Q, K, V = q[a:b, hd], k[ka:kb, hd // group], v[ka:kb, hd // group]
                x = scale * (Q @ K.T)
                X = U * (d + 4) * scale * (Q.abs() @ K.abs().T) + 4 * U * x.abs()
                if bias is not None:
                    add = bias[:, hd][row]
                    x = x + add
                    X = X + torch.where(add.isfinite(), 4 * U * (add.abs() + x.abs()), 0.0)
                seen = (rel <= 0) if causal else torch.ones_like(rel, dtype=torch.bool)
                x = x.masked_fill(~seen, -math.inf)
                X = torch.where(x == -math.inf, 0.0, X)
                top = x.max(1, keepdim=True).values
                ref = torch.where(top == -math.inf, torch.zeros_like(top), top)
                e = torch.exp(x - ref)
                total = e.sum(1, keepdim=True)
                p = torch.where(total > 0, e / total, torch.zeros_like(e))
                g = 2 * X.max(1, keepdim=True).values + 8 * U
                lse = (ref + torch.log(total))[:, 0]
                self.lse[hd, a:b] = lse
                tol["lse"][hd, a:b] = (g + n * U)[:, 0] + 4 * U * torch.nan_to_num(lse.abs(), posinf=0.0)
                out, wide = p @ V, p @ V.abs()
                e_out = (p_step + g + n * U) * wide
                self.out[a:b, hd] = out
                tol["out"][a:b, hd] = e_out + h * out.abs()
                if dout is None:
                    continue
                do = dout[a:b, hd].double()
                dp, delta = do @ V.T, (do * out).sum(1, keepdim=True)
                ds = p * (dp - delta)
                e_delta = (do.abs() * (e_out + kept * (out.abs() + e_out))).sum(1, keepdim=True) + \
                    (d + 4) * U * (do.abs() * out.abs()).sum(1, keepdim=True)
                e_ds = (g + (d + 4) * U) * p * (do.abs() @ V.abs().T + delta.abs()) + p * e_delta
                e_ds = e_ds + 4 * U * ds.abs()
                take = h * (ds.abs() + e_ds) + e_ds
                dk, dv = scale * (ds.T @ Q), p.T @ do
                self.dq[a:b, hd] = scale * (ds @ K)
                self.dk[ka:kb, hd // group] += dk
                self.dv[ka:kb, hd // group] += dv
                tol["dq"][a:b, hd] = scale * ((take + n * U * ds.abs()) @ K.abs())
                m = (b - a) * group
                tol["dk"][ka:kb, hd // group] += scale * ((take + m * U * ds.abs()).T @ Q.abs())
                tol["dv"][ka:kb, hd // group] += (p * (h + g + m * U)).T @ do.abs()
                if bias is not None:
                    count = lambda t: torch.bincount(row.reshape(-1), t.reshape(-1), len(bias))  # noqa: E731
                    self.dbias[:, hd] += count(ds)
                    tol["dbias"][:, hd] += count(e_ds + n * (b - a) * U * ds.abs())
        for n in ("dq", "dk", "dv"):
            tol[n] += 2 * h * getattr(self, n).abs()
        if bias is not None:
            tol["dbias"] += 2 * bias_step * self.dbias.abs()
        self.tol, self.grads = tol, dout is not None

    def check(self, got):
        """`got`: name -> tensor.  Every element within its bound (and 1e-30)."""
        for name, x in got.items():
            want, tol = getattr(self, name), self.tol[name]
            assert x.shape == want.shape, name
            x = x.double()
            bad = torch.where(want.isfinite(), ~((x - want).abs() <= tol + 1e-30), x != want)
            if bad.any():
                i = tuple(int(j) for j in bad.nonzero()[0])
                raise AssertionError(f"{name}: {int(bad.sum())} of {x.numel()} elements beyond their "
                                     f"bound, first {i}: {float(x[i])} for {float(want[i])} +- "
                                     f"{float(tol[i])}")
