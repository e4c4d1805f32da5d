"""Calls of one handle that are in work at the same time, on two streams without a wait between them, each with its own workspace: the same bits as
one after the other."""
import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200.configs import CrossAttentionConfig, LayerNormConfig

pytestmark = pytest.mark.gpu


def at_once(calls, results):
    """`calls` one after the other, then each on a stream of its own, all of them held back by one event until the last is in its queue."""
    for c in calls:
        c()
    torch.cuda.synchronize()
    want = [t.clone() for t in results]
    streams, gate = [torch.cuda.Stream() for _ in calls], torch.cuda.Event()
    slow = torch.zeros(1 << 27, device="cuda")
    for _ in range(3):
        for t in results:
            t.fill_(float("nan"))
        for _ in range(40):
            slow.add_(1.0)                                   # (some milliseconds, while the calls below are queued)
        gate.record()
        for _ in range(4):
            for s, c in zip(streams, calls):
                s.wait_event(gate)
                with torch.cuda.stream(s):
                    c()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, want))


def test_layer_norm():
    d = 1000
    norm, calls, results = B.LayerNorm(LayerNormConfig(d)), [], []
    for i, tokens in enumerate((3000, 2000, 37)):
        gen = torch.Generator("cuda").manual_seed(i)
        x, dy = (torch.randn(2, tokens, d, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
        w = torch.randn(d, generator=gen, device="cuda")
        y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)

        def call(x=x, w=w, dy=dy, y=y, dx=dx, dw=dw, db=db):
            norm.forward(x, w, w, y)
            norm.backward(x, w, dy, dx, dw, db)
        calls.append(call)
        results += [y, dx, dw, db]
    at_once(calls, results)


def test_cross_attention():
    """Keys in parts joined by a second launch, queries and keys in parts backward, and the few-rows kernel."""
    a, calls, results = B.CrossAttention(CrossAttentionConfig(64, 4, 2)), [], []
    for i, (N, K) in enumerate(((200, 3000), (3000, 200), (260, 2000), (2, 1000))):
        gen = torch.Generator("cuda").manual_seed(i)
        q, dout = (torch.randn(1, 4, N, 64, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
        k, v = (torch.randn(1, 2, K, 64, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
        out, dq, dk, dv = (torch.empty_like(t) for t in (q, q, k, v))
        lse = torch.empty(1, 4, N, device="cuda")

        def call(q=q, k=k, v=v, out=out, lse=lse, dout=dout, dq=dq, dk=dk, dv=dv):
            a.forward(q, k, v, out, lse)
            a.backward(q, k, v, out, lse, dout, dq, dk, dv)
        calls.append(call)
        results += [out, lse, dq, dk, dv]
    at_once(calls, results)
    assert a.device_status() == 0
