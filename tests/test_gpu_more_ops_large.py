"""Attention and AdamW where places pass 32 bits."""
import numpy as np
import pytest

import adamw_ref as ref

pytestmark = pytest.mark.gpu


def test_attention_over_a_long_cache():
    """k, v and their gradients of 4.3e9 elements each; the last head, whose elements lie
    furthest, of a query over 2^20 keys and of the sequence behind it."""
    import torch
    import paper_1909_08029_amd as rip
    from attn_ref import Attention
    heads, dim, nq, nk = 16, 256, 301, (1 << 20) + 700
    assert nk * heads * dim > 1 << 32
    gen = torch.Generator(device="cuda").manual_seed(2)
    make = lambda n: torch.randn(n, heads, dim, generator=gen, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    q, k, v, dout = make(nq), make(nk), make(nk), make(nq)
    qo, ko = [0, 1, nq], [0, 1 << 20, nk - 50]
    o, p = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (qo, ko))
    out, kept = rip.rip_attn_forward(q, k, v, o, p)
    dq, dk, dv = rip.rip_attn_backward(dout, q, k, v, out, kept, o, p)
    assert (dk[-50:] == 0).all() and (dv[-50:] == 0).all()
    h = slice(heads - 1, heads)
    Attention(q[:, h], k[:, h], v[:, h], qo, ko, dout=dout[:, h]).check(
        dict(out=out[:, h], lse=kept.lse[h], dq=dq[:, h], dk=dk[:, h], dv=dv[:, h]))


def test_adamw_of_more_than_two_to_the_32():
    """The last elements before and after 2^32 of one segment, to the bit."""
    import torch
    import paper_1909_08029_amd as rip
    n, seed, step = (1 << 32) + 4133, 77, 3
    gen = torch.Generator(device="cuda").manual_seed(3)
    h = dict(lr=1e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1, grad_scale=1.0)
    param, grad = (torch.empty(n, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    for t in (param, grad):
        for part in t.split(1 << 28):
            part.copy_(torch.randn(len(part), generator=gen, device="cuda", dtype=torch.bfloat16))
    state = rip.AdamwState.zeros(rip.Replicas([[param]], [[grad]]), 8)
    spans = [(0, 4096), ((1 << 32) - 4096, 1 << 32), (1 << 32, n)]
    before = [param[a:b].float().cpu().numpy() for a, b in spans]
    rip.rip_adamw_step(state, [0], step, seed=seed, **h)
    key = ref.key_of(seed, step, 0, 0)
    for (a, b), w in zip(spans, before):
        g, z = grad[a:b].float().cpu().numpy(), np.zeros(b - a, np.float32)
        w, m, v = ref.update(w, g, z, z, step, h["lr"], *h["betas"], h["eps"], h["weight_decay"], 1.0)
        assert a >> 32 == (b - 1) >> 32
        k = (key + (a >> 32) * 0x9E3779B9) & 0xffffffff
        rnd = ref.hashes_from(a & 0xffffffff, b - a, k)
        e0, e1 = a // 32, -(-b // 32)
        for got, want in zip((param[a:b].view(torch.int16), state.m[0][0][a:e1 * 32], state.m_exps[0][0][e0:e1],
                              state.v[0][0][a:e1 * 32], state.v_exps[0][0][e0:e1]),
                             (ref.to_bf16(w).view(np.int16), *ref.encode_m(m, rnd), *ref.encode_v(v, rnd))):
            np.testing.assert_array_equal(got.cpu().numpy(), want)
