"""The operators on a stream of their own, in a captured graph, and with a
workspace that holds leftovers."""
import pytest

from train_ops_ref import BF16

pytestmark = pytest.mark.gpu


def state(seed):
    import torch
    torch.manual_seed(seed)
    tokens, vocab, width, inner = 600, 777, 136, 72
    r = lambda *s: torch.randn(*s, device="cuda").to(BF16)  # noqa: E731
    ids = torch.randint(-1, vocab, (tokens,), device="cuda")
    return dict(table=r(vocab, width), ids=ids, dout=r(tokens, width), gate=r(tokens, inner),
                up=r(tokens, inner), dh=r(tokens, inner), x=r(tokens, width), dy=r(tokens, inner),
                logits=r(tokens, vocab), targets=ids.clone(),
                offsets=torch.tensor([0, 100, 250, 400, 600], dtype=torch.int32, device="cuda"),
                ref=torch.randn(4, device="cuda") - 900, old=torch.randn(tokens, device="cuda") - 7,
                adv=torch.randn(tokens, device="cuda"),
                table_grad=torch.empty(vocab, width, device="cuda"),
                weight_grad=torch.empty(inner, width, device="cuda"),
                g1=torch.empty(tokens, vocab, device="cuda", dtype=BF16),
                g2=torch.empty(tokens, vocab, device="cuda", dtype=BF16))


def every_call(rip, s, stream=None):
    out = [rip.rip_embed_lookup(s["table"], s["ids"], 2.0, stream=stream),
           rip.rip_embed_grad(s["dout"], s["ids"], s["table_grad"], 2.0, stream=stream)]
    h, g8, u8 = rip.rip_gate_forward(s["gate"], s["up"], stream=stream)
    dg, du, h8 = rip.rip_gate_backward(s["dh"], g8, u8, hidden=True, stream=stream)
    out += [h, dg, du, rip.rip_ckpt_unpack(h8, stream=stream)]
    x8 = rip.rip_ckpt_pack(s["x"], stream=stream)
    out.append(rip.rip_ckpt_wgrad(s["dy"], x8, s["weight_grad"], stream=stream))
    out += rip.rip_pref_loss(s["logits"], s["targets"], s["offsets"], s["ref"], 0.1, 0.1,
                             grad=s["g1"], stream=stream)
    out += rip.rip_policy_loss(s["logits"], s["targets"], s["old"], s["adv"], grad=s["g2"],
                               stream=stream)
    return out + [s["g1"], s["g2"]]


def test_on_another_stream():
    import torch
    import paper_1909_08029_amd as rip
    want = [t.clone() for t in every_call(rip, state(1))]
    s = state(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = every_call(rip, s, stream=side)
    del s["x"]                      # freed memory may be handed out again on this stream
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    with torch.cuda.stream(side):   # and where that stream is torch's current one
        got = every_call(rip, state(1))
    side.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)


def test_in_a_graph():
    import torch
    import paper_1909_08029_amd as rip
    s = state(2)
    every_call(rip, s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = every_call(rip, s)
    for seed in (2, 3, 4, 3):
        new = state(seed)
        for k in s:
            s[k].copy_(new[k])
        g.replay()
        torch.cuda.synchronize()
        want = every_call(rip, new)
        for i, (a, b) in enumerate(zip(out, want)):
            assert torch.equal(a, b), (seed, i)


def test_workspaces_need_not_be_clear():
    import ctypes
    import torch
    import paper_1909_08029_amd as rip
    s = state(5)
    for n in (600, 5000):
        ids = torch.randint(0, 40, (n,), device="cuda")
        dout = torch.randn(n, 136, device="cuda")
        nbytes = rip.lib.rip_embed_grad_workspace(n, 136)
        got = []
        for fill in (0, 255):
            ws = torch.full((nbytes,), fill, dtype=torch.uint8, device="cuda")
            grad = torch.empty(777, 136, device="cuda")
            assert rip.lib.rip_embed_grad(dout.data_ptr(), 0, 136, ids.data_ptr(), 1, n, 1.0,
                                          grad.data_ptr(), 0, 777, 136, 136, 0, ws.data_ptr(),
                                          nbytes, ctypes.c_void_p(rip._stream_ptr(None))) == 0
            got.append(grad)
        assert torch.equal(*got)
    nbytes = rip.lib.rip_pref_loss_workspace(600, 777, 2)
    got = []
    for fill in (0, 255):
        ws = torch.full((nbytes,), fill, dtype=torch.uint8, device="cuda")
        out, grad = torch.empty(1 + 4, device="cuda"), torch.empty_like(s["logits"])
        p = out.data_ptr()
        assert rip.lib.rip_pref_loss(s["logits"].data_ptr(), 1, 777, 600, 777,
                                     s["targets"].data_ptr(), 1, s["offsets"].data_ptr(), 2,
                                     s["ref"].data_ptr(), 0.1, 0.0, 1.0, p, p + 4, None,
                                     grad.data_ptr(), 777, ws.data_ptr(), nbytes,
                                     ctypes.c_void_p(rip._stream_ptr(None))) == 0
        got += [out, grad]
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[3])
