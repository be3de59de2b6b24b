"""Performance cases of the attention between a language-model replica's embedding
and its loss, with a learned relative position bias, and of the AdamW update of
replicas before their P-Reduce.

Each case is one pass through an operator, in the plain form (elementary torch
operations in 32 bits, rounded once) or, with ``own``, through the framework's
entry points.

A case's fields:
  kind      "attend"  attention without anything kept: every sequence has `rows`
                      queries, the last of its ragged keys (sampling between
                      training steps)
            "train"   attention of packed sequences and its backward pass
            "bias"    the same with a learned relative position bias by buckets,
                      and the bias's gradient
            "adamw"   the AdamW update of replicas of many tensors; states of 8
                      bits are read back as values in the same pass
  tokens    rows of k and v; elements of one replica (adamw)
  seqs      packed sequences; tensors of a replica (adamw)
  rows      queries of a sequence (attend); replicas (adamw)
  heads, kv, dim    heads of q, heads of k and v, width of a head
  causal    queries see no later keys
  buckets, far, both    rows of the bias table, the distance from which on all
                      keys share a row, and whether later keys have rows of
                      their own
  dtype     "f32" or "bf16": activations; parameters and gradients (adamw)
  store     "f32" or "bf16": the bias table and its gradient
  bits      32 or 8: AdamW's states

Distances from a query to a key (key - query) fall into intervals: those of up to
`buckets` / 2 (a half of that with `both`) have a row each, the others rows whose
widths grow by a constant factor up to `far`.

AdamW's states in 8 bits are held in blocks of 32 elements.  The first moment is
q * 2^e, q in -127..127, e as small as the block's largest magnitude allows
(at least -126).  The second is f * 2^e, f = y for a code 16 x + y with x = 0,
else (16 + y) * 2^(x - 1); the largest f is 31 * 2^14, and a positive value has a
code above 0.  Both round up with the probability that keeps the mean, by 16
random bits each, a hash of the element's index.
"""
import functools
import math
import random

import torch

own = False

LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
STEP, GRAD_SCALE, SEED = 100, 0.5, 12345
BLOCK = 32
TOP = 31 << 14                      # largest f of a second moment in 8 bits


def _case(name, kind, tokens, seqs=1, rows=0, heads=0, kv=0, dim=0, causal=True, buckets=0, far=0,
          both=False, dtype="bf16", store="bf16", bits=32):
    case = dict(kind=kind, tokens=tokens, seqs=seqs, rows=rows, heads=heads, kv=kv, dim=dim,
                causal=causal, buckets=buckets, far=far, both=both, dtype=dtype, store=store,
                bits=bits)
    return dict(case, name=name) if name else case


def listed():
    return [
        # one decoding step of a handful of sampled sequences between training
        # steps; latency
        _case("attend_8x1", "attend", 5000, 8, 1, 16, 16, 64),
        # a decoding step after long prompts: few queries, a long axis of keys
        _case("attend_4x1_200k", "attend", 200_003, 4, 1, 32, 8, 128),
        # three short sequences in fp32 with an odd head width (a test's size); latency
        _case("train_101_f32", "train", 101, 3, heads=3, kv=3, dim=40, dtype="f32"),
        # shared heads in fp32, two sequences
        _case("train_2k_f32", "train", 2049, 2, heads=8, kv=2, dim=72, dtype="f32"),
        # a micro-batch of sixteen pairs of ragged length, width 1024
        _case("train_8k_bf16", "train", 8192, 32, heads=16, kv=16, dim=64),
        # one long sequence of a model of 1.3 G parameters (width 2048), shared heads
        _case("train_16k_bf16", "train", 16_384, 1, heads=16, kv=4, dim=128),
        # an encoder's bias over two odd sequences in fp32; latency
        _case("bias_37_f32", "bias", 37, 2, heads=2, kv=2, dim=24, causal=False, buckets=8, far=20,
              both=True, dtype="f32", store="f32"),
        # an encoder's micro-batch: fp32 storage, bf16 activations
        _case("bias_8k_bf16", "bias", 8192, 16, heads=16, kv=16, dim=64, causal=False, buckets=32,
              far=128, both=True, store="f32"),
        # a long sequence of a decoder, all bf16
        _case("bias_8k_causal", "bias", 8192, 1, heads=16, kv=16, dim=128, buckets=32, far=1024),
        # four replicas of a small model of five tensors; latency
        _case("adamw_98k_f32", "adamw", 97_664, 5, 4, dtype="f32"),
        # four replicas of 25.6 M parameters in many tensors, states of 32 bits
        _case("adamw_25m_f32", "adamw", 25_600_000, 161, 4, dtype="f32"),
        # one bf16 replica of 1.3 G parameters, states of 8 bits
        _case("adamw_1g3_8bit", "adamw", 1_300_000_000, 290, 1, bits=8),
    ]


def _size(rng, lo, hi):
    """A size spread over the logarithm of lo..hi, odd ones among them."""
    n = int(round(lo * (hi / lo) ** rng.random()))
    if rng.random() < 0.3 and n >= 128:
        n = n // 64 * 64
    return min(hi, max(lo, n))


def draw(rng):
    kind = rng.choice(["attend", "train", "train", "bias", "bias", "adamw"])
    if kind == "adamw":
        replicas = rng.choice([1, 1, 2, 4])
        return _case("", kind, _size(rng, 1000, 100_000_000 // replicas), _size(rng, 1, 300),
                     replicas, dtype=rng.choice(["f32", "bf16"]), bits=rng.choice([32, 8]))
    dtype = rng.choice(["f32", "bf16", "bf16"])
    kv = _size(rng, 1, 16)
    heads = min(32 // kv, rng.choice([1, 1, 2, 4, 8])) * kv
    dim = rng.choice([32, 64, 64, 80, 128, 128, 256, _size(rng, 8, 256)])
    if kind == "attend":
        seqs, rows = _size(rng, 1, 32), rng.choice([1, 1, 1, 4, 16])
        tokens = _size(rng, seqs * 3 * rows, min(200_003, (1 << 30) // (heads * seqs * rows),
                                                 (1 << 28) // (heads * dim)))
        return _case("", kind, tokens, seqs, rows, heads, kv, dim, dtype=dtype)
    most = math.isqrt(((1 << 28) if dtype == "f32" else (1 << 30)) // heads)
    tokens = _size(rng, 8, min(8192, most))
    case = dict(heads=heads, kv=kv, dim=dim, dtype=dtype, causal=rng.random() < 0.6)
    if kind == "bias":
        case.update(buckets=rng.choice([8, 16, 32, 32, 64]), far=_size(rng, 40, 1000),
                    both=not case["causal"], store=rng.choice(["f32", "bf16"]))
    return _case("", kind, tokens, _size(rng, 1, min(32, tokens // 4)), **case)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _normal(gen, shape, dtype, sigma=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype).mul_(sigma)


def _cuts(total, parts, seed, least):
    """`parts` ragged lengths of at least `least` that add up to `total`."""
    rng = random.Random(seed)
    share = [rng.uniform(0.3, 1.7) for _ in range(parts)]
    scale, at, ends = (total - least * parts) / sum(share), 0.0, []
    for x in share:
        at += x * scale
        ends.append(int(round(at)))
    return [b - a + least for a, b in zip([0] + ends, ends)]


@functools.lru_cache(maxsize=64)
def _tensors(total, n):
    """(size, place) of a replica's tensors in a flat buffer, a few large ones and
    many small ones, each at a multiple of 32, and the buffer's size."""
    rng = random.Random(n)
    share = [math.exp(rng.gauss(0, 2)) for _ in range(n)]
    sizes = [max(1, int(total * x / sum(share))) for x in share]
    sizes[sizes.index(max(sizes))] += total - sum(sizes)
    places, at = [], 0
    for x in sizes:
        places.append((x, at))
        at += -(-x // BLOCK) * BLOCK
    return places, at


def _edges(rows, far):
    """Smallest distance of each of `rows` rows: half of them take a distance each,
    the others grow by a constant factor up to `far` (in exact integers)."""
    exact = rows // 2
    steps, edges, n = rows - exact, list(range(exact)), exact
    for i in range(steps):
        while n ** steps < exact ** (steps - i) * far ** i:
            n += 1
        edges.append(n)
    return edges


@functools.lru_cache(maxsize=64)
def _intervals(buckets, far, both):
    """(first distance of every interval but the lowest, row of each interval) of
    key - query, ascending."""
    half = buckets // 2 if both else buckets
    edges = _edges(half, far)
    starts, rows = [], [half - 1]
    for b in range(half - 1, 0, -1):       # earlier keys, from far to near
        if edges[b] == (edges[b + 1] if b + 1 < half else None):
            rows[-1] = b - 1
            continue
        starts.append(1 - edges[b])
        rows.append(b - 1)
    for b in range(1, half) if both else ():
        if edges[b] == (edges[b + 1] if b + 1 < half else None):
            continue
        starts.append(edges[b])
        rows.append(half + b)
    return tuple(starts), tuple(rows)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, tokens, act = case["kind"], case["tokens"], _TYPES[case["dtype"]]
    s = dict(case=case)
    if kind == "adamw":
        places, flat = _tensors(tokens, case["seqs"])
        sigma = torch.zeros(flat, device="cuda")       # a tensor's gradients have a size of their own
        for i, (n, at) in enumerate(places):
            sigma[at:at + n] = 1e-3 * (1 + i % 7)
        shape = (case["rows"], flat)
        s["param"] = _normal(gen, shape, act, 0.02).mul_(sigma > 0)
        s["grad"] = _normal(gen, shape, act).mul_(sigma)
        s["m"] = _normal(gen, shape, torch.float32, 0.1).mul_(sigma)       # some steps old
        s["v"] = _normal(gen, shape, torch.float32, 0.2).mul_(sigma).square_()
        if case["bits"] == 8:  # codes and exponents
            half = torch.full((), 0.5, device="cuda")
            for name, encode in (("m", _encode_m), ("v", _encode_v)):
                codes, exps = encode(s[name].view(-1, BLOCK), half)
                s[name], s[name + "_exps"] = codes.view(shape), exps.view(shape[0], -1)
        if own:
            import paper_1909_08029_amd as rip
            cut = lambda x, unit=1: [[row[at // unit:-(-(at + n) // unit)] for n, at in places]  # noqa: E731
                                     for row in x]
            rep = rip.Replicas(cut(s["param"]), cut(s["grad"]))
            if case["bits"] == 32:
                s["adamw"] = rip.AdamwState(rep, cut(s["m"]), cut(s["v"]))
            else:  # whole blocks of codes
                codes = [[[row[at:at + -(-n // BLOCK) * BLOCK] for n, at in places] for row in s[x]]
                         for x in ("m", "v")]
                s["adamw"] = rip.AdamwState(rep, *codes, cut(s["m_exps"], BLOCK),
                                            cut(s["v_exps"], BLOCK))
        return s
    heads, kv, dim, seqs = case["heads"], case["kv"], case["dim"], case["seqs"]
    lengths = _cuts(tokens, seqs, seed, max(1, case["rows"]))
    ends = torch.tensor([0] + lengths, device="cuda").cumsum(0).to(torch.int32)
    s["k_offsets"] = ends
    if kind == "attend":
        s["q_offsets"] = torch.arange(seqs + 1, device="cuda", dtype=torch.int32) * case["rows"]
        queries = seqs * case["rows"]
    else:
        s["q_offsets"], queries = ends, tokens
        s["dout"] = _normal(gen, (queries, heads, dim), act, 1e-3)
    s["q"] = _normal(gen, (queries, heads, dim), act, 1.4)
    s["k"] = _normal(gen, (tokens, kv, dim), act, 1.4)
    s["v"] = _normal(gen, (tokens, kv, dim), act)
    if kind == "bias":
        s["bias"] = _normal(gen, (case["buckets"], heads), _TYPES[case["store"]])
        s["dbias"] = torch.zeros_like(s["bias"])
        s["buckets"] = _intervals(case["buckets"], case["far"], case["both"])
        if own:
            import paper_1909_08029_amd as rip
            s["buckets"] = rip.RelBuckets(*s["buckets"])
        else:
            s["starts"] = torch.tensor(s["buckets"][0], device="cuda")
            s["of"] = torch.tensor(s["buckets"][1], device="cuda")
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    import paper_1909_08029_amd as rip
    case = s["case"]
    kind, causal = case["kind"], case["causal"]
    if kind == "adamw":
        state = s["adamw"]
        rip.rip_adamw_step(state, range(case["rows"]), STEP, LR, (BETA1, BETA2), EPS, DECAY,
                           grad_scale=GRAD_SCALE, seed=SEED)
        if case["bits"] == 32:
            return s["param"], s["m"], s["v"]
        return s["param"], *state.moments(torch.bfloat16)
    if kind == "attend":
        return rip.rip_attn_forward(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"],
                                    causal=causal, keep=False)[0]
    bias, buckets = s.get("bias"), s.get("buckets")
    out, kept = rip.rip_attn_forward(s["q"], s["k"], s["v"], s["q_offsets"], causal=causal,
                                     bias=bias, buckets=buckets)
    grads = rip.rip_attn_backward(s["dout"], s["q"], s["k"], s["v"], out, kept, s["q_offsets"],
                                  causal=causal, bias=bias, buckets=buckets, dbias=s.get("dbias"))
    return (out, kept.lse, *grads) if bias is None else (out, kept.lse, *grads, s["dbias"])


def _hash(index, key):
    """The 32-bit finalizer of MurmurHash3 over index ^ key."""
    x = index ^ key
    x = ((x ^ (x >> 16)) * 0x85ebca6b) & 0xffffffff
    x = ((x ^ (x >> 13)) * 0xc2b2ae35) & 0xffffffff
    return x ^ (x >> 16)


def _mix64(x):
    """SplitMix64's output function."""
    x = ((x ^ (x >> 30)) * 0xBF58476D1CE4E5B9) % (1 << 64)
    x = ((x ^ (x >> 27)) * 0x94D049BB133111EB) % (1 << 64)
    return x ^ (x >> 31)


def _key(step, replica, tensor):
    """The hash's key: seed, step, replica and tensor folded in turn."""
    k = SEED
    for c in (step, replica, tensor):
        k = _mix64((k + 0x9E3779B97F4A7C15 * (c + 1)) % (1 << 64))
    return k & 0xffffffff


def _two_to(e):
    return ((e + 127) << 23).view(torch.float32)


def _value_m(codes, exps):
    return codes.float() * _two_to(exps.int() - 127)[:, None]


def _value_v(codes, exps):
    c = codes.int()
    x, y = c >> 4, c & 15
    f = torch.where(x == 0, y, (16 + y) << (x - 1).clamp(min=0))
    return f.float() * _two_to(exps.int() - 127)[:, None]


def _exponent(x, top, least=-126):
    """Smallest e of which top * 2^e reaches the largest magnitude of each block."""
    f, e = torch.frexp(x.abs().amax(1))            # largest = f * 2^e, 0.5 <= f < 1
    t, k = math.frexp(top)
    e = torch.where(f <= t, e - k, e - k + 1)
    return torch.where(f == 0, torch.full_like(e, least), e).clamp(min=least)


def _encode_m(x, r):
    e = _exponent(x, 127)
    q = torch.floor(x * _two_to(-e)[:, None] + r).clamp(-127, 127)
    return q.to(torch.int8), (e + 127).to(torch.uint8)


def _encode_v(x, r):
    e = _exponent(x, TOP)
    t = x * _two_to(-e)[:, None]
    low = torch.floor(t + r).int()
    bits = t.view(torch.int32) + (r * 65536).int() * 8
    code = torch.where(t < 16, low, (bits >> 19) - (130 << 4))
    code = torch.maximum(code, (x > 0).int())
    return code.clamp(max=255).to(torch.uint8), (e + 127).to(torch.uint8)


def _plain_adamw(s):
    case = s["case"]
    decay = 1 - LR * DECAY
    rate, root = LR / (1 - BETA1 ** STEP), 1 / math.sqrt(1 - BETA2 ** STEP)
    g = s["grad"].float() * GRAD_SCALE
    m, v = s["m"], s["v"]
    if case["bits"] == 8:
        m = _value_m(m.view(-1, BLOCK), s["m_exps"].view(-1)).view(g.shape)
        v = _value_v(v.view(-1, BLOCK), s["v_exps"].view(-1)).view(g.shape)
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * (1 - BETA2) * g
    del g
    s["param"].copy_(s["param"].float() * decay - m * rate / (torch.sqrt(v) * root + EPS))
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return s["param"], s["m"], s["v"]
    places, _ = _tensors(case["tokens"], case["seqs"])
    out_m, out_v = torch.empty_like(s["param"]).bfloat16(), torch.empty_like(s["param"]).bfloat16()
    for r in range(case["rows"]):
        for t, (n, at) in enumerate(places):
            whole = slice(at, at + -(-n // BLOCK) * BLOCK)
            h = _hash(torch.arange(whole.stop - at, device="cuda"), _key(STEP, r, t))
            for name, x, bits, out, encode, value in (
                    ("m", m, h & 0xffff, out_m, _encode_m, _value_m),
                    ("v", v, h >> 16, out_v, _encode_v, _value_v)):
                codes, exps = encode(x[r, whole].view(-1, BLOCK), bits.float().div_(65536).view(-1, BLOCK))
                s[name][r, whole] = codes.view(-1)
                s[name + "_exps"][r, at // BLOCK:whole.stop // BLOCK] = exps
                out[r, whole] = value(codes, exps).view(-1)
    return s["param"], out_m, out_v


def _place(offsets, n):
    """Of each of n rows: its sequence, and its distance from the sequence's end."""
    at = torch.arange(n, device="cuda")
    seq = torch.searchsorted(offsets, at, right=True, out_int32=True) - 1
    return seq, at - offsets[1:].long()[seq.long()]


def _run_plain(s):
    case = s["case"]
    if case["kind"] == "adamw":
        return _plain_adamw(s)
    heads, kv, act = case["heads"], case["kv"], _TYPES[case["dtype"]]
    group, scale = heads // kv, case["dim"] ** -0.5
    q = s["q"].float().transpose(0, 1)
    k, v = (s[n].float().repeat_interleave(group, 1).transpose(0, 1) for n in ("k", "v"))
    (q_seq, q_at), (k_seq, k_at) = (_place(s[n + "_offsets"], len(s[n])) for n in ("q", "k"))
    hidden = q_seq[:, None] != k_seq[None, :]
    if case["causal"]:
        hidden |= k_at[None, :] > q_at[:, None]
    p = torch.matmul(q, k.transpose(1, 2)).mul_(scale)
    if case["kind"] == "bias":
        far = torch.bucketize(k_at[None, :] - q_at[:, None], s["starts"], right=True)
        p += s["bias"].float().t()[:, s["of"][far]]
    p.masked_fill_(hidden, -math.inf)
    top = p.amax(2, keepdim=True)
    p = p.sub_(top).exp_()
    total = p.sum(2, keepdim=True)
    p /= total
    out = torch.matmul(p, v).transpose(0, 1).to(act)
    if case["kind"] == "attend":
        return out
    lse = (top + torch.log(total))[:, :, 0]
    dout = s["dout"].float().transpose(0, 1)
    shared = lambda x: x.view(kv, group, -1, case["dim"]).sum(1).transpose(0, 1).to(act)  # noqa: E731
    dv = shared(torch.matmul(p.transpose(1, 2), dout))
    ds = torch.matmul(dout, v.transpose(1, 2))
    ds -= (ds * p).sum(2, keepdim=True)
    ds *= p
    del p
    dq = (torch.matmul(ds, k) * scale).transpose(0, 1).to(act)
    dk = shared(torch.matmul(ds.transpose(1, 2), q) * scale)
    if case["kind"] == "train":
        return out, lse, dq, dk, dv
    # keys at one distance lie on a diagonal; rows of twice the width, one element
    # short, put each of them into a column
    n = case["tokens"]
    wide = torch.nn.functional.pad(ds.flip(1), (0, n)).view(heads, -1)[:, :-n]
    along = wide.reshape(heads, n, 2 * n - 1).sum(1, dtype=torch.float64)
    far = torch.bucketize(torch.arange(1 - n, n, device="cuda"), s["starts"], right=True)
    dbias = torch.zeros((heads, case["buckets"]), dtype=torch.float64, device="cuda")
    dbias.index_add_(1, s["of"][far], along)
    return out, lse, dq, dk, dv, dbias.t().to(s["bias"].dtype).contiguous()


# ---------------------------------------------------------------------------
def _pairs(case):
    """Pairs of a query and a key that it sees."""
    if case["kind"] == "attend":
        return case["tokens"] * case["rows"]
    lengths = _cuts(case["tokens"], case["seqs"], 0, 1)
    return sum(n * (n + 1) // 2 if case["causal"] else n * n for n in lengths)


def work(case):
    size = {"f32": 4, "bf16": 2}
    a, n = size[case["dtype"]], case["tokens"]
    if case["kind"] == "adamw":  # states of 8 bits: codes, a byte a block, and the values read back
        state = 8 if case["bits"] == 32 else 2 + 2 / BLOCK
        n *= case["rows"]
        return {"bytes": int(n * (3 * a + 2 * state + (0 if case["bits"] == 32 else 4))),
                "flops": 14 * n}
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    queries = case["seqs"] * case["rows"] if case["kind"] == "attend" else n
    q, k = queries * heads * dim * a, n * kv * dim * a
    pairs = _pairs(case) * heads
    if case["kind"] == "attend":
        return {"bytes": 2 * q + 2 * k, "flops": pairs * (4 * dim + 5)}
    # forward: q, k, v in, out and the rows' sums out; backward: those and dout in,
    # three gradients out
    return {"bytes": 6 * q + 6 * k + 8 * queries * heads, "flops": pairs * (14 * dim + 15)}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_attention(case, s):
    heads, group, dim = case["heads"], case["heads"] // case["kv"], case["dim"]
    cuts = list(zip(*(s[n].tolist() for n in ("q_offsets", "k_offsets"))))
    need = case["kind"] != "attend"
    zeros = lambda x: torch.zeros(x.shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out, dq, dk, dv = zeros(s["q"]), zeros(s["q"]), zeros(s["k"]), zeros(s["v"])
    lse = torch.zeros((heads, len(s["q"])), dtype=torch.float64, device="cuda")
    dbias = zeros(s["bias"]) if "bias" in s else None
    for (a, ka), (b, kb) in zip(cuts, cuts[1:]):
        if a == b:
            continue
        ahead = (kb - ka) - (b - a) + torch.arange(b - a, device="cuda")
        rel = torch.arange(kb - ka, device="cuda")[None, :] - ahead[:, None]
        if dbias is not None:
            row = torch.zeros_like(rel)
            starts, rows = s["intervals"]
            row += rows[0]
            for first, r in zip(starts, rows[1:]):
                row[rel >= first] = r
        for h in range(heads):
            q, k, v = s["q"][a:b, h], s["k"][ka:kb, h // group], s["v"][ka:kb, h // group]
            q, k, v = (x.double().contiguous().requires_grad_(need) for x in (q, k, v))
            x = torch.mm(q, k.t()) / math.sqrt(dim)
            if dbias is not None:
                add = s["bias"][:, h].double()[row].requires_grad_()
                x = x + add
            if case["causal"]:
                x = x.masked_fill(rel > 0, -math.inf)
            o = torch.mm(torch.softmax(x, 1), v)
            out[a:b, h], lse[h, a:b] = o.detach(), torch.logsumexp(x.detach(), 1)
            if need:
                o.backward(s["dout"][a:b, h].double())
                dq[a:b, h] = q.grad
                dk[ka:kb, h // group] += k.grad
                dv[ka:kb, h // group] += v.grad
            if dbias is not None:
                dbias[:, h] += torch.bincount(row.view(-1), add.grad.view(-1), case["buckets"])
    if not need:
        return out
    return (out, lse, dq, dk, dv) if dbias is None else (out, lse, dq, dk, dv, dbias)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] != "adamw":
        if case["kind"] == "bias":
            s["intervals"] = _intervals(case["buckets"], case["far"], case["both"])
        return _exact_attention(case, s)
    m, v = s["m"].double(), s["v"].double()
    if case["bits"] == 8:
        x = torch.div(v, 16, rounding_mode="floor")
        v = torch.where(x > 0, (16 + v % 16) * torch.exp2(x - 1), v)
        del x
        m *= torch.exp2(s["m_exps"].double() - 127).repeat_interleave(BLOCK, 1)
        v *= torch.exp2(s["v_exps"].double() - 127).repeat_interleave(BLOCK, 1)
    g = GRAD_SCALE * s["grad"].double()
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g ** 2
    del g
    w = s["param"].double()
    w -= LR * (m / (1 - BETA1 ** STEP) / ((v / (1 - BETA2 ** STEP)).sqrt() + EPS) + DECAY * w)
    # a state of 8 bits is a random rounding of these
    return (w, m, v) if case["bits"] == 32 else (w, None, None)
