"""AdamW as the replicas' local update, to the bit against numpy."""
import ctypes

import numpy as np
import pytest

import adamw_ref as ref

pytestmark = pytest.mark.gpu

SIZES = [1, 31, 32, 0, 33, 2048, 2049, 7001]
HYPER = dict(lr=3e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1, grad_scale=0.5, seed=(1 << 63) + 5)


def values(t):
    """float32 values of a tensor."""
    return t.float().cpu().numpy()


class Setup:
    def __init__(self, dtype, bits, sizes=SIZES, n=3, seed=0, odd=0, zeros=False):
        import torch
        import paper_1909_08029_amd as rip
        gen = torch.Generator(device="cuda").manual_seed(seed)
        t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        self.sizes, self.n, self.bits, self.dtype = sizes, n, bits, dtype
        total = sum(sizes) + odd

        def make(sigma):
            out = []
            for _ in range(n):
                flat = (torch.randn(total, generator=gen, device="cuda") * sigma).to(t)
                at, row = odd, []
                for s in sizes:   # back to back: segments begin anywhere
                    row.append(flat[at:at + s])
                    at += s
                out.append(row)
            return out
        if odd == 0:
            self.param, self.grad = make(0.02), make(1e-3)
            self.rep = rip.Replicas(self.param, self.grad)
        else:   # 16-byte aligned segments in buffers of their own
            pad = lambda rows: [[s.clone() for s in row] for row in rows]  # noqa: E731
            self.param, self.grad = pad(make(0.02)), pad(make(1e-3))
            self.rep = rip.Replicas(self.param, self.grad)
        self.state = rip.AdamwState.zeros(self.rep, bits)
        if zeros:
            return
        for r in range(n):
            for s, size in enumerate(sizes):
                m = torch.randn(size, generator=gen, device="cuda") * 1e-4
                v = (torch.randn(size, generator=gen, device="cuda") * 2e-4) ** 2
                if bits == 32:
                    self.state.m[r][s].copy_(m)
                    self.state.v[r][s].copy_(v)
                else:
                    h = np.full(size, 0x80008000, np.uint32)
                    for name, x, enc in (("m", m, ref.encode_m), ("v", v, ref.encode_v)):
                        c, e = enc(x.cpu().numpy(), h)
                        getattr(self.state, name)[r][s].copy_(torch.from_numpy(c))
                        getattr(self.state, name + "_exps")[r][s].copy_(torch.from_numpy(e))

    def snapshot(self):
        get = lambda rows: [[x.clone() for x in row] for row in rows]  # noqa: E731
        s = self.state
        return [get(x) for x in (self.param, s.m, s.v, s.m_exps, s.v_exps) if x is not None]

    def expected(self, before, r, s, step, h):
        """Arrays of one segment after a step: param as stored, m, v (codes, exps)."""
        w, g = values(before[0][r][s]), values(self.grad[r][s])
        if self.bits == 32:
            m, v = values(before[1][r][s]), values(before[2][r][s])
        else:
            m = ref.value_m(before[1][r][s].cpu().numpy(), before[3][r][s].cpu().numpy())[:len(w)]
            v = ref.value_v(before[2][r][s].cpu().numpy(), before[4][r][s].cpu().numpy())[:len(w)]
        w, m, v = ref.update(w, g, m, v, step, h["lr"], *h["betas"], h["eps"], h["weight_decay"],
                             h["grad_scale"])
        if self.dtype == "bf16":
            w = (ref.to_bf16(w).astype(np.uint32) << np.uint32(16)).view(np.float32)
        if self.bits == 32:
            return [w, m, v]
        rnd = ref.hashes(len(w), ref.key_of(h["seed"], step, r, s))
        (mc, me), (vc, ve) = ref.encode_m(m, rnd), ref.encode_v(v, rnd)
        return [w, mc, vc, me, ve]

    def check(self, before, after, active, step, h):
        for r in range(self.n):
            for s in range(len(self.sizes)):
                got = [x[r][s] for x in after]
                if r in active:
                    want = self.expected(before, r, s, step, h)
                    got = [values(got[0])] + [x.cpu().numpy() for x in got[1:]]
                    for a, b in zip(got, want):
                        np.testing.assert_array_equal(a, b, err_msg=f"replica {r} segment {s}")
                else:
                    assert all((a == x[r][s]).all() for a, x in zip(got, before))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("odd", [0, 1])
def test_steps(dtype, bits, odd):
    import paper_1909_08029_amd as rip
    x = Setup(dtype, bits, odd=odd)
    for step, active in ((1, [0, 2]), (2, [1]), (1000, [2, 0, 1]), (1001, [])):
        before = x.snapshot()
        rip.rip_adamw_step(x.state, active, step, **HYPER)
        x.check(before, x.snapshot(), active, step, HYPER)


@pytest.mark.parametrize("bits", [32, 8])
def test_extremes(bits):
    """Gradients from nothing to infinity: blocks of zeros, subnormals, squares
    beyond fp32, NaN; each stays in its block."""
    import torch
    import paper_1909_08029_amd as rip
    x = Setup("f32", bits, sizes=[32 * 12], n=1, zeros=True)
    g = x.grad[0][0].view(12, 32)
    g[0] = 0
    g[1] = 1e-30
    g[2] = 1e-42
    g[3] = torch.logspace(-22, 3, 32)
    g[4] = 1e18
    g[5, 7] = 1e25           # its square is an infinity
    g[6, 3] = float("inf")
    g[7, 9] = float("nan")
    g[8] = 3e38
    g[9] = torch.logspace(-4, 0, 32)
    g[10] = -1
    for step in (1, 2, 3):
        before = x.snapshot()
        rip.rip_adamw_step(x.state, [0], step, **HYPER)
        x.check(before, x.snapshot(), [0], step, HYPER)


def test_roots_of_all_magnitudes():
    """Second moments from far below the smallest normal number to 2^100, waves of one
    magnitude, of all, and with zeros among them; eps so small that the root counts."""
    import torch
    import paper_1909_08029_amd as rip
    h = dict(HYPER, eps=1e-37, weight_decay=0.0, grad_scale=1.0)
    x = Setup("f32", 8, sizes=[1 << 18, 1 << 16, 6145], n=1)
    gen = torch.Generator(device="cuda").manual_seed(9)
    for k, g in enumerate(x.grad[0]):
        power = torch.randint(-74, 51, (len(g),), generator=gen, device="cuda")
        if k == 0:                                  # a power for each 512 elements
            power = power[:len(g) // 512].repeat_interleave(512)
        g.copy_((1 + torch.rand(len(g), generator=gen, device="cuda")) * 2.0 ** power.float())
        if k == 2:
            g[torch.rand(len(g), generator=gen, device="cuda") < 0.01] = 0
    for step in (1, 2):
        before = x.snapshot()
        rip.rip_adamw_step(x.state, [0], step, **h)
        x.check(before, x.snapshot(), [0], step, h)


def test_roundings_keep_the_mean():
    """A second moment that shrinks by 0.1% a step, between codes 3 to 6% apart, and a
    first moment of a few steps of its block follow their exact values on average."""
    import torch
    import paper_1909_08029_amd as rip
    n, steps = 32 * 2048, 400
    x = Setup("f32", 8, sizes=[n], n=1, zeros=True)
    x.grad[0][0].zero_()
    m, v = np.full(n, 3e-4, np.float32), np.full(n, 3e-7, np.float32)
    m[::32], v[::32] = 1e-2, 1e-4             # the blocks' largest values
    h = np.full(n, 0x80008000, np.uint32)
    (mc, me), (vc, ve) = ref.encode_m(m, h), ref.encode_v(v, h)
    for t, a in ((x.state.m, mc), (x.state.v, vc), (x.state.m_exps, me), (x.state.v_exps, ve)):
        t[0][0].copy_(torch.from_numpy(a))
    m0, v0 = (t.double() for t in x.state.moments())
    for step in range(1, steps + 1):
        rip.rip_adamw_step(x.state, [0], step, lr=0.0, betas=(0.99, 0.999), seed=7)
    m1, v1 = (t.double() for t in x.state.moments())
    small = (torch.arange(n, device="cuda") % 32 != 0)
    # The sum over 63488 elements of a code that moves by one in a few steps: each
    # step's rounding errs by at most one step with a variance of at most 1/4, and
    # later decay only shrinks it, so the mean of 63488 errs by a standard deviation of
    # at most sqrt(400 / 4 / 63488) = 0.04 steps of that code; 6 of them are 0.24.
    want_m = float(m0[0][small].mean()) * 0.99 ** steps
    assert abs(float(m1[0][small].mean()) - want_m) < 0.24 * 2.0 ** (int(me[0]) - 127)
    want_v = float(v0[0][small].mean()) * 0.999 ** steps
    assert abs(float(v1[0][small].mean()) / want_v - 1) < 0.24 / 16


def test_moments_layout():
    import torch
    x = Setup("bf16", 8)
    for dtype in (torch.float32, torch.bfloat16):
        m, v = x.state.moments(dtype)
        at = 0
        for s, size in enumerate(SIZES):
            whole = -(-size // 32) * 32
            for r in range(x.n):
                for out, value, kind in ((m, ref.value_m, "m"), (v, ref.value_v, "v")):
                    want = value(getattr(x.state, kind)[r][s].cpu().numpy(),
                                 getattr(x.state, kind + "_exps")[r][s].cpu().numpy())
                    np.testing.assert_array_equal(values(out[r, at:at + whole]), want)
            at += whole
        assert m.shape == v.shape == (x.n, at)


@pytest.mark.parametrize("bits", [32, 8])
def test_replayed_graph_with_scalars_on_the_device(bits):
    import torch
    import paper_1909_08029_amd as rip
    live, eager = Setup("bf16", bits), Setup("bf16", bits)
    scalars = rip.rip_adamw_scalars(1, **HYPER).cuda()
    stream = torch.cuda.Stream()
    start = [[[t.clone() for t in row] for row in kind] for kind in live.snapshot()]
    with torch.cuda.stream(stream):
        rip.rip_adamw_step(live.state, [0, 1], 1, scalars=scalars, **HYPER)   # warm
    stream.synchronize()
    now = (live.param, live.state.m, live.state.v, live.state.m_exps, live.state.v_exps)
    for kind, saved in zip([k for k in now if k is not None], start):
        for row, old in zip(kind, saved):
            for t, o in zip(row, old):
                t.copy_(o)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rip.rip_adamw_step(live.state, [0, 1], 1, scalars=scalars, **HYPER)
    for step in (1, 2, 3, 17):
        h = dict(HYPER, lr=1e-3 * step)
        scalars.copy_(rip.rip_adamw_scalars(step, **h))
        graph.replay()
        rip.rip_adamw_step(eager.state, [0, 1], step, **h)
        torch.cuda.synchronize()
        for a, b in zip(live.snapshot(), eager.snapshot()):
            for p, q in zip(a, b):
                assert all(torch.equal(y, z) for y, z in zip(p, q))


def test_refusals():
    import torch
    import paper_1909_08029_amd as rip
    x = Setup("f32", 8, sizes=[64, 64])
    step = lambda **k: rip.rip_adamw_step(x.state, **dict(dict(active=[0], step=1, lr=1e-3), **k))  # noqa: E731
    for change in (dict(step=0), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=0.0),
                   dict(eps=1e-60), dict(lr=float("nan")), dict(weight_decay=float("inf")),
                   dict(active=[3]), dict(active=[-1]), dict(active=[1, 1]), dict(active=[0, 1, 2, 0])):
        with pytest.raises(rip.RipError):
            step(**change)
    with pytest.raises(ValueError):
        step(scalars=torch.zeros(6))                       # not on the device
    with pytest.raises(ValueError):
        step(scalars=torch.zeros(5, device="cuda"))
    with pytest.raises(ValueError):
        rip.AdamwState(rip.Replicas(x.param), x.state.m, x.state.v)   # no gradients
    with pytest.raises(ValueError):
        rip.AdamwState(x.rep, x.state.m, x.state.v)        # codes without exponents
    with pytest.raises(ValueError):
        rip.AdamwState(x.rep, x.state.m[:2], x.state.v, x.state.m_exps, x.state.v_exps)
    with pytest.raises(rip.RipError) as e:                 # moments that share memory
        m = [[torch.zeros(64, device="cuda")] * 2 for _ in range(3)]
        rip.AdamwState(x.rep, m, [[torch.zeros(64, device="cuda") for _ in r] for r in m])
    assert e.value.code == rip.RIP_E_OVERLAP
    with pytest.raises(rip.RipError) as e:                 # codes at any address
        off = [[torch.zeros(100, dtype=torch.int8, device="cuda")[1:65] for _ in range(2)] for _ in range(3)]
        rip.AdamwState(x.rep, off, x.state.v, x.state.m_exps, x.state.v_exps)
    assert e.value.code == rip.RIP_E_ALIGN
    with pytest.raises(rip.RipError) as e:
        Setup("f32", 32).state.moments()                   # nothing to decode
    assert e.value.code == rip.RIP_E_UNSUPPORTED
    buf = torch.zeros(3 * 128 * 4, device="cuda")
    rc = rip.lib.rip_adamw_moments(x.state._h, 0, buf.data_ptr(), buf.data_ptr() + 64, None)
    assert rc == rip.RIP_E_OVERLAP
    rc = rip.lib.rip_adamw_moments(x.state._h, 0, x.param[0][0].data_ptr(), buf.data_ptr(), None)
    assert rc == rip.RIP_E_OVERLAP
    assert ctypes.sizeof(rip._adamw._Scalars) == 24


def test_before_a_p_reduce():
    """A step of the algorithm with AdamW in place of SGD."""
    import torch
    import paper_1909_08029_amd as rip
    x, y = Setup("f32", 8), Setup("f32", 8)
    rip.rip_adamw_step(x.state, [0, 1, 2], 5, **HYPER)
    rip.rip_preduce(x.rep, [[0, 2]])
    before = y.snapshot()
    want = [[y.expected(before, r, s, 5, HYPER)[0] for s in range(len(SIZES))] for r in range(3)]
    for s in range(len(SIZES)):
        mean = (want[0][s] + want[2][s]) * np.float32(0.5)
        for r, expect in ((0, mean), (1, want[1][s]), (2, mean)):
            np.testing.assert_array_equal(values(x.param[r][s]), expect)
    torch.cuda.synchronize()
