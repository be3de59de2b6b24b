"""Attention, its relative position bias and its backward pass against 64-bit
references, every element within the bound of its roundings (attn_ref)."""
import math

import pytest

from attn_ref import Attention

pytestmark = pytest.mark.gpu


def tensors(dtype, heads, kv, dim, nq, nk, seed=0, pad=0):
    """q, k, v, dout; with `pad` the rows are parts of wider ones."""
    import torch
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def make(n, h):
        x = torch.randn(n, h * dim + pad, generator=gen, device="cuda").to(t)
        return x[:, pad // 2:pad // 2 + h * dim].unflatten(1, (h, dim))
    return make(nq, heads), make(nk, kv), make(nk, kv), make(nq, heads)


def offsets(values):
    import torch
    return None if values is None else torch.tensor(values, dtype=torch.int32, device="cuda")


def run(q, k, v, dout, qo, ko=None, causal=True, scale=None, bias=None, buckets=None, dbias=None, **kw):
    """name -> tensor of a forward and a backward pass."""
    import torch
    import paper_1909_08029_amd as rip
    args = dict(causal=causal, scale=scale, bias=bias, buckets=buckets)
    out, kept = rip.rip_attn_forward(q, k, v, offsets(qo), offsets(ko), **args)
    if bias is not None and dbias is None:
        dbias = torch.full_like(bias, float("nan"))
    dq, dk, dv = rip.rip_attn_backward(dout, q, k, v, out, kept, offsets(qo), offsets(ko), dbias=dbias,
                                       **args, **kw)
    got = dict(out=out, lse=kept.lse, dq=dq, dk=dk, dv=dv)
    return got if bias is None else dict(got, dbias=dbias)


def against(q, k, v, dout, qo, ko=None, causal=True, scale=None, bias=None, buckets=None):
    got = run(q, k, v, dout, qo, ko, causal, scale, bias, buckets)
    rel = {} if bias is None else dict(bias=bias, starts=buckets.starts, rows=buckets.rows)
    Attention(q, k, v, qo, ko, causal, scale, dout=dout, **rel).check(got)
    return got


# sequences of none, one and many tokens, borders of tiles, tokens before and behind all
PACKED = [0, 0, 1, 33, 33, 97, 225, 226, 290]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [1, 8, 31, 64, 72, 96, 128, 136, 255, 256])
@pytest.mark.parametrize("causal", [True, False])
def test_head_dims(dtype, dim, causal):
    against(*tensors(dtype, 2, 1, dim, 290, 290), PACKED, causal=causal)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (6, 2), (5, 1), (32, 4)])
def test_shared_heads(dtype, heads, kv):
    against(*tensors(dtype, heads, kv, 40, 300, 300), [3, 70, 295])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("qo,ko", [
    ([0, 1, 2, 3], [0, 500, 1501, 1502]),         # single queries, a long axis of keys
    ([0, 16, 20], [0, 2000, 2100]),
    ([0, 70, 70, 200], [0, 20, 90, 95]),          # more queries than keys: rows that see none
    ([0, 130, 131], [0, 0, 600]),                 # no keys at all
    ([0, 0, 64], [0, 64, 64]),                    # keys without queries
])
def test_other_lengths_of_keys(dtype, causal, qo, ko):
    against(*tensors(dtype, 4, 2, 64, qo[-1] + 2, ko[-1] + 5), qo, ko, causal)


@pytest.mark.parametrize("dtype,heads,kv,dim,lengths", [
    ("bf16", 2, 2, 64, [2500]), ("bf16", 2, 1, 128, [1200, 900]), ("f32", 1, 1, 128, [1500]),
    ("bf16", 1, 1, 256, [1100]), ("bf16", 8, 8, 64, [300] * 12), ("f32", 2, 2, 64, [700, 650]),
])
def test_long(dtype, heads, kv, dim, lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    for causal in (True, False):
        against(*tensors(dtype, heads, kv, dim, at[-1], at[-1]), at, causal=causal)


def table(buckets, heads, dtype="f32", seed=1):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(buckets, heads, generator=gen, device="cuda")
    return x if dtype == "f32" else x.bfloat16()


@pytest.mark.parametrize("dtype,store", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("buckets,far,both", [(32, 128, True), (8, 20, True), (16, 1000, False), (64, 40, False)])
@pytest.mark.parametrize("causal", [True, False])
def test_bias(dtype, store, buckets, far, both, causal):
    import paper_1909_08029_amd as rip
    against(*tensors(dtype, 2, 2, 64, 700, 700), [0, 0, 5, 420, 421, 690], causal=causal,
            bias=table(buckets, 2, store), buckets=rip.RelBuckets.log(buckets, far, both))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [24, 128, 200])
def test_bias_with_shared_heads_and_other_keys(dtype, dim):
    import paper_1909_08029_amd as rip
    b = rip.RelBuckets.log(16, 90, True)
    against(*tensors(dtype, 6, 2, dim, 300, 700), [0, 100, 299], [0, 60, 690], False, bias=table(16, 6), buckets=b)
    against(*tensors(dtype, 4, 1, dim, 40, 1500), [0, 1, 40], [0, 900, 1500], True, bias=table(16, 4), buckets=b)


@pytest.mark.parametrize("starts,rows", [
    ([], [0]),                                           # one bucket
    ([0], [1, 0]),
    ([-3], [0, 0]),                                      # intervals that share a row
    ([-40, 0, 1, 41], [2, 1, 0, 1, 2]),                  # symmetric
    ([5000], [0, 1]),                                    # never reached
    ([-5001, -5000], [0, 1, 1]),
    ([-1023, 1023], [0, 2, 1]),                          # the widest span
    (list(range(-63, 64)), [i % 5 for i in range(128)]),  # as many as there may be
])
def test_intervals(starts, rows):
    import paper_1909_08029_amd as rip
    for dtype in ("f32", "bf16"):
        against(*tensors(dtype, 1, 1, 32, 500, 500), [0, 60, 500], causal=False, bias=table(7, 1),
                buckets=rip.RelBuckets(starts, rows))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [64, 80, 128, 256])
@pytest.mark.parametrize("span", [1468, 1469, 2048])
def test_wide_spans(dtype, dim, span):
    """Sums of many distances in LDS beside the tiles, at every width; one and many tiles."""
    import paper_1909_08029_amd as rip
    first = 1 - span // 2
    b = rip.RelBuckets([first, -3, 0, first + span - 2], [3, 1, 0, 2, 4])
    against(*tensors(dtype, 2, 1, dim, 1301, 1301), [0, 1200, 1301], causal=False, bias=table(5, 2), buckets=b)


def test_a_bias_that_hides_keys():
    """-inf in the table is a mask; queries that it leaves nothing have zeros."""
    import torch
    import paper_1909_08029_amd as rip
    for dtype in ("f32", "bf16"):
        x = tensors(dtype, 2, 2, 64, 400, 400)
        bias = table(3, 2)
        bias[0] = -math.inf                              # a window of 50 keys back ...
        bias[2, 1] = -math.inf                           # ... and for head 1 none ahead
        against(*x, [0, 10, 400], causal=False, bias=bias, buckets=rip.RelBuckets([-50, 1], [0, 1, 2]))
        bias = torch.full((2, 2), -math.inf, device="cuda")
        bias[1, 0] = 3.0                                 # head 0 sees far keys only, head 1 none
        got = against(*x, [0, 10, 400], causal=True, bias=bias, buckets=rip.RelBuckets([-99], [1, 0]))
        for name in ("out", "dq", "dk", "dv"):
            assert (got[name][:, 1] == 0).all()
        assert (got["lse"][1] == -math.inf).all() and (got["lse"][0, 10:109] == -math.inf).all()
        assert (got["dbias"][:, 1] == 0).all()
        low = torch.finfo(torch.float32).min             # as some programs write a mask
        bias = torch.tensor([[low, 0.5], [1.0, low]], device="cuda")
        against(*x, [0, 10, 400], causal=True, bias=bias, buckets=rip.RelBuckets([-20], [0, 1]))
        for big in (-60000.0, 3000.0):                   # still a bias
            against(*x, [0, 10, 400], causal=True, bias=torch.full((2, 2), big, device="cuda"),
                    buckets=rip.RelBuckets([-20], [0, 1]))


def test_what_other_sequences_hold():
    """Infinities and NaN in one sequence, and in tokens of none, reach no other."""
    import torch
    for dtype in ("f32", "bf16"):
        x = tensors(dtype, 2, 1, 64, 300, 300)
        for t in x:
            t[40:90] = float("nan")
            t[50] = float("inf")
            t[:3] = float("nan")
            t[291:] = float("inf")
        got = run(*x, [3, 40, 90, 291])
        for t in x:
            t[40:90] = 0
            t[:3] = 0
            t[291:] = 0
        want = run(*x, [3, 40, 90, 291])
        for name in ("out", "dq", "dk", "dv"):
            for part in (slice(0, 40), slice(90, 300)):
                assert torch.equal(got[name][part], want[name][part])
            assert not got[name][40:90].isfinite().all()   # not lost either
        assert torch.equal(got["lse"][:, 90:], want["lse"][:, 90:])


def test_offsets_out_of_order():
    import torch
    x = tensors("bf16", 2, 2, 32, 200, 200)
    for bad in ([5, 3, 80, 60, 500], [-9, 100, 100, 20, 150], [300, 0, 10]):
        against(*x, bad)
    ok = tensors("f32", 1, 1, 16, 200, 150)
    against(*ok, [0, 90, 80, 250], [10, 5, 400, 100])
    assert torch.cuda.is_available()


@pytest.mark.parametrize("sequences", [2, 1100])
def test_one_list_for_both_sides(sequences):
    """The same tensor as both offsets, with other numbers of queries and keys: it is cut
    to each side's tokens."""
    import paper_1909_08029_amd as rip
    import torch
    at = [0, 90, 200] if sequences == 2 else [0] * (sequences - 1) + [90, 200]
    o = offsets(at)
    for dtype in ("f32", "bf16"):
        for nq, nk in ((200, 150), (120, 200)):
            q, k, v, dout = tensors(dtype, 2, 1, 64, nq, nk)
            out, kept = rip.rip_attn_forward(q, k, v, o, o, causal=False)
            dq, dk, dv = rip.rip_attn_backward(dout, q, k, v, out, kept, o, o, causal=False)
            Attention(q, k, v, at, at, causal=False, dout=dout).check(
                dict(out=out, lse=kept.lse, dq=dq, dk=dk, dv=dv))
    assert torch.cuda.is_available()


def test_many_sequences():
    """More than every workgroup puts in order by itself; one and two tokens each."""
    at = [0]
    for i in range(1500):
        at.append(at[-1] + 1 + i % 2)
    x = tensors("bf16", 2, 1, 32, at[-1] + 7, at[-1] + 7)
    got = run(*x, at)
    # sequences of one token: p is 1
    import torch
    ones = torch.tensor([a for a, b in zip(at, at[1:]) if b - a == 1], device="cuda")
    assert torch.equal(got["out"][ones], x[2][ones].expand(-1, 2, -1))
    Attention(*[t[:90] for t in x[:3]], at[:61], dout=x[3][:90]).check({k: (v[:, :90] if k == "lse" else v[:90])
                                                                       for k, v in got.items()})
    assert (got["out"][at[-1]:] == 0).all() and (got["dk"][at[-1]:] == 0).all()
    at[700], at[701] = at[701], at[700]            # and out of order
    bad = run(*x, at)
    k = list(at)
    assert bad["out"].isfinite().all() and k


def test_strides_and_scale():
    for dtype in ("f32", "bf16"):
        x = tensors(dtype, 3, 3, 31, 150, 150, pad=9)
        against(*x, [0, 150], scale=0.37)
        against(*x, [0, 150], causal=False, scale=1e-6)
        against(*x, [1, 2, 149], scale=4.0)


def test_parts_of_one_buffer():
    """q, k and v side by side in a projection's rows, gradients likewise, heads of
    odd width; what lies between is left alone."""
    import torch
    heads, kv, dim, n = 4, 2, 13, 170
    for t in (torch.float32, torch.bfloat16):
        buf = torch.randn(n, (heads + 2 * kv) * dim + 3, device="cuda").to(t)
        cut = lambda b: [b[:, i * dim:j * dim].unflatten(1, (j - i, dim))  # noqa: E731
                         for i, j in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv))]
        q, k, v = cut(buf)
        dout = torch.randn(n, heads, dim, device="cuda").to(t)
        gbuf = torch.full_like(buf, 7.0)
        dq, dk, dv = cut(gbuf)
        got = run(q, k, v, dout, [0, 100, 170], dq=dq, dk=dk, dv=dv)
        assert got["dq"] is dq
        Attention(q, k, v, [0, 100, 170], dout=dout).check(got)
        assert (gbuf[:, -3:] == 7).all()


def test_bias_gradient_added():
    import torch
    import paper_1909_08029_amd as rip
    for store in ("f32", "bf16"):
        x = tensors("bf16", 2, 2, 64, 300, 300)
        bias, b = table(8, 2, store), rip.RelBuckets.log(8, 20)
        first = run(*x, [0, 300], causal=False, bias=bias, buckets=b)["dbias"]
        again = torch.ones_like(bias)
        run(*x, [0, 300], causal=False, bias=bias, buckets=b, dbias=again, accumulate=True)
        # one more rounding of the sum
        step = 2.0 ** -8 if store == "bf16" else 2.0 ** -24
        want = first.double() + 1
        assert ((again.double() - want).abs() <= 2 * step * (want.abs() + first.double().abs())).all()
        wide = torch.full((8, 5), 3.0, device="cuda")     # a table's columns among others
        args = dict(causal=False, bias=wide[:, 1:3], buckets=b)
        grad = torch.full_like(wide, 9.0)
        run(*x, [0, 300], dbias=grad[:, 1:3], **args)
        assert (grad[:, 0] == 9).all() and (grad[:, 3:] == 9).all() and grad[:, 1:3].abs().max() < 9


def test_gradients_by_differences():
    """The loss sum(out * dout) moves by the gradients: central differences of the
    64-bit definition in random directions."""
    import torch
    import paper_1909_08029_amd as rip
    q, k, v, dout = tensors("f32", 2, 1, 24, 90, 90, seed=3)
    bias, b, at = table(8, 2), rip.RelBuckets.log(8, 20, True), [0, 37, 90]
    got = run(q, k, v, dout, at, causal=False, bias=bias, buckets=b)
    loss = lambda *x: float((Attention(x[0], x[1], x[2], at, causal=False, bias=x[3], starts=b.starts,  # noqa: E731
                                       rows=b.rows).out * dout.double()).sum())
    base = [t.double() for t in (q, k, v, bias)]
    for i, name in enumerate(("dq", "dk", "dv", "dbias")):
        d = torch.randn_like(base[i])
        eps = 1e-5
        up, down = ([t + s * eps * d if j == i else t for j, t in enumerate(base)] for s in (1, -1))
        slope, mine = (loss(*up) - loss(*down)) / (2 * eps), float((got[name].double() * d).sum())
        assert abs(slope - mine) <= 1e-4 * float((got[name].double().abs() * d.abs()).sum()), name


def test_same_bits_every_time():
    import torch
    import paper_1909_08029_amd as rip
    x = tensors("bf16", 4, 2, 64, 900, 900)
    bias, b = table(32, 4), rip.RelBuckets.log(32, 128, False)
    runs = [run(*x, [0, 600, 900], bias=bias, buckets=b) for _ in range(3)]
    for got in runs[1:]:
        for name, t in got.items():
            assert torch.equal(t, runs[0][name]), name


def test_streams_graphs_and_dirty_workspaces():
    import torch
    import paper_1909_08029_amd as rip
    x = tensors("bf16", 4, 2, 64, 40, 3000)
    bias, b = table(32, 4), rip.RelBuckets.log(32, 128, True)
    qo, ko = offsets([0, 10, 40]), offsets([0, 1000, 3000])
    args = dict(causal=True, bias=bias, buckets=b)

    def both(stream=None):
        out, kept = rip.rip_attn_forward(*x[:3], qo, ko, **args, stream=stream)
        db = torch.empty_like(bias)
        return [out, kept.lse, *rip.rip_attn_backward(x[3], *x[:3], out, kept, qo, ko, **args, dbias=db,
                                                      stream=stream), db]
    want = [t.clone() for t in both()]
    junk = torch.full((1 << 26,), float("nan"), device="cuda")   # what the allocator hands out next
    del junk
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for seed in (0, 5, 6):
        for t, new in zip(x, tensors("bf16", 4, 2, 64, 40, 3000, seed=seed)):
            t.copy_(new)
        graph.replay()
        eager = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(held, eager))


def test_autograd_sees_what_is_written():
    import torch
    import paper_1909_08029_amd as rip
    q, k, v, dout = tensors("f32", 1, 1, 16, 20, 20)
    q.requires_grad_()
    out = torch.zeros_like(q.detach())
    got, kept = rip.rip_attn_forward(q, k, v, offsets([0, 20]), out=out)
    assert got is out and not got.requires_grad and out._version > 0
    dq = torch.zeros_like(out)
    rip.rip_attn_backward(dout, q, k, v, out, kept, offsets([0, 20]), dq=dq)
    assert dq._version > 0


def test_empty():
    import torch
    import paper_1909_08029_amd as rip
    for nq, nk, at in ((0, 0, [0]), (0, 5, [0, 0]), (5, 0, [0, 0]), (4, 4, [0]), (0, 0, [0, 0, 0])):
        x = tensors("bf16", 2, 1, 32, nq, nk)
        bias, b = table(4, 2), rip.RelBuckets([-1, 0, 1], [0, 1, 2, 3])
        got = run(*x, at, [0] * len(at), bias=bias, buckets=b)
        assert all((t == 0).all() for n, t in got.items() if n != "lse")
        assert (got["lse"] == -math.inf).all()
    torch.cuda.synchronize()


def test_refusals_of_the_binding():
    import torch
    import paper_1909_08029_amd as rip
    q, k, v, dout = tensors("bf16", 4, 2, 16, 20, 20)
    at, b = offsets([0, 20]), rip.RelBuckets([0], [0, 1])
    out, kept = rip.rip_attn_forward(q, k, v, at)
    fwd = lambda **c: rip.rip_attn_forward(**dict(dict(q=q, k=k, v=v, q_offsets=at), **c))  # noqa: E731
    for bad in (dict(q=q.float()), dict(q=q[:, :, :8]), dict(k=k[:, :1]), dict(v=v[:10]), dict(q=q.transpose(0, 1)),
                dict(q=q.view(20, 64)), dict(k=k.cpu()), dict(q_offsets=at.long()),
                dict(q_offsets=at[:0]), dict(k_offsets=offsets([0, 1, 2])), dict(bias=table(2, 4)),
                dict(buckets=b), dict(bias=table(2, 3), buckets=b), dict(out=out.float()),
                dict(out=out[:, :2]), dict(q=q[:, ::2])):
        with pytest.raises((ValueError, TypeError)):
            fwd(**bad)
    for bad in (dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(q=q[:, :3].contiguous()),
                dict(q=q[:10]), dict(bias=table(1, 4), buckets=b), dict(out=q)):
        with pytest.raises(rip.RipError):
            fwd(**bad)
    bwd = lambda **c: rip.rip_attn_backward(**dict(dict(dout=dout, q=q, k=k, v=v, out=out, kept=kept,  # noqa: E731
                                                        q_offsets=at), **c))
    for bad in (dict(kept=rip.Kept(kept.lse[:2], kept.low)), dict(kept=rip.Kept(kept.lse.double(), None)),
                dict(kept=rip.Kept(kept.lse, out.float())), dict(dbias=table(2, 4)),
                dict(dq=q.float()), dict(dk=q), dict(bias=table(2, 4), buckets=b, dbias=table(3, 4))):
        with pytest.raises((ValueError, TypeError)):
            bwd(**bad)
    for bad in (dict(dq=q), dict(dk=k), dict(dv=v), dict(dq=dout)):
        with pytest.raises(rip.RipError) as e:
            bwd(**bad)
        assert e.value.code == rip.RIP_E_OVERLAP
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nq,nk", [(0, 600), (600, 0), (0, 5000), (5000, 0)])
def test_one_empty_side(dtype, dim, nq, nk):
    """Queries without keys and keys without queries, more than a split is made for: every
    row of every output is written, with zeros (log-sums: -inf)."""
    import torch
    import paper_1909_08029_amd as rip
    q, k, v, dout = tensors(dtype, 4, 2, dim, nq, nk)
    at = [0, nq // 2, nq], [0, nk // 3, nk]
    bias, b = table(4, 4), rip.RelBuckets([-1, 0, 1], [0, 1, 2, 3])
    for args in (dict(), dict(bias=bias, buckets=b)):
        grads = [torch.full_like(t, float("nan")) for t in (q, k, v)]
        got = run(q, k, v, dout, *at, **args, dq=grads[0], dk=grads[1], dv=grads[2])
        for name, t in got.items():
            assert (t == (-math.inf if name == "lse" else 0)).all(), name
    kept = torch.full_like(bias, 3.0)
    run(q, k, v, dout, *at, bias=bias, buckets=b, dbias=kept, accumulate=True)
    assert (kept == 3).all()
