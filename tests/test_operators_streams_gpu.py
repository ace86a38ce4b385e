"""The stream of a call that names none: the one that torch has current."""
import pytest
import torch

import paper_2004_08771_amd as hb

pytestmark = pytest.mark.gpu

B, K = 64, 300


class Calls:
    """All operators on one input, into buffers of their own."""

    def __init__(self):
        g = torch.Generator(device="cuda").manual_seed(3)
        self.y = torch.randint(0, K, (B,), device="cuda", generator=g, dtype=torch.int32)
        self.row, self.seq = torch.randn(B, device="cuda", generator=g), torch.tensor([0, 20, 64], dtype=torch.int32, device="cuda")
        new = lambda *s: torch.full(s, 7.0, device="cuda")  # noqa: E731
        self.out, self.d1, self.d2, self.d3 = new(B, K), new(B, K), new(B, K), new(B, K)
        self.lp, self.lse, self.s1, self.s2 = new(B), new(B), new(4), new(4)
        self.ws = [torch.zeros(hb.choice_workspace_bytes(B, 1), dtype=torch.uint8, device="cuda") for _ in range(3)]

    def run(self, Z, **stream):
        hb.dropout(Z, self.out, 0.3, 1, **stream)
        hb.logprob(Z, self.y, self.lp, self.lse, ws=self.ws[0], **stream)
        hb.logprob_grad(Z, self.y, self.lp, self.lse, self.row, self.d1, **stream)
        hb.policy_loss(Z, self.y, self.lp, self.row, self.s1, dZ=self.d2, ws=self.ws[1], **stream)
        hb.preference_loss(Z, self.y, self.seq, self.s2, dZ=self.d3, ws=self.ws[2], **stream)

    def results(self):
        return [t.clone() for t in (self.out, self.lp, self.lse, self.d1, self.s1, self.d2, self.s2, self.d3)]


def test_calls_follow_the_current_stream():
    """The input is made on that stream, behind half a second of products: a call on another one would read what was there before."""
    want, got = Calls(), Calls()
    big = torch.zeros(8192, 8192, device="cuda", dtype=torch.bfloat16)
    src = torch.randn(B, K, device="cuda")
    Z = torch.zeros(B, K, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for _ in range(400):
            big = big @ big
        Z.copy_(src)
        got.run(Z)
        done = got.results()
    s.synchronize()
    want.run(src)
    want.run(src, stream=0)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(done, want.results()))


def test_calls_are_captured_on_the_current_stream():
    want, got = Calls(), Calls()
    Z = torch.randn(B, K, device="cuda")
    got.run(Z)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got.run(Z)
    for k in range(4):
        Z.normal_()
        for t in (got.out, got.d1, got.d2, got.d3, got.lp, got.s1, got.s2):
            t.fill_(float(k))
        g.replay()
        want.run(Z)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got.results(), want.results())), k
