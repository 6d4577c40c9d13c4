"""The operators of the two ends together with those between, captured and replayed, on other streams, several at once."""
import numpy as np
import pytest

import ends_ref as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import paper_2001_00532_amd as psk  # noqa: E402


class Model:
    """Tokens -> rows of a shared table in 8 bits -> a layer of a mixture of experts -> logits by the same table."""

    def __init__(self, n, seed):
        g = torch.Generator().manual_seed(seed)
        self.n, self.vocab, self.dim, inter, experts = n, 500, 144, 64, 6
        w = torch.randn(self.vocab, self.dim, generator=g)
        self.codes, self.scales = torch.empty((self.vocab, self.dim), dtype=torch.int8, device="cuda"), torch.empty(self.vocab, device="cuda")
        psk.psk_quant_i8(w.cuda(), self.codes, self.scales)
        self.table = psk.I8(self.codes, self.scales)
        self.router = (torch.randn(experts, self.dim, generator=g) / 12).half().cuda()
        self.w1, self.w3 = ((torch.randn(experts, inter, self.dim, generator=g) / 12).half().cuda() for _ in range(2))
        self.w2 = (torch.randn(experts, self.dim, inter, generator=g) / 8).half().cuda()
        self.x, self.z = (torch.empty(n, self.dim, dtype=torch.float16, device="cuda") for _ in range(2))
        self.crd, self.vals = torch.empty(n, 2, dtype=torch.int32, device="cuda"), torch.empty(n, 2, device="cuda")
        self.logits = torch.empty(n, self.vocab, dtype=torch.float16, device="cuda")
        self.grad = torch.empty(self.vocab, self.dim, device="cuda")
        self.ws = [psk.psk_moe_route_workspace(n, experts), psk.psk_moe_workspace(n, self.dim, inter, experts, 2), psk.psk_linear_i8_workspace(self.table, self.z),
                   psk.psk_embed_grad_workspace(self.z, self.grad)]
        self.ids = torch.randint(-1, self.vocab, (n,), generator=g, dtype=torch.int32).cuda()

    def run(self):
        psk.psk_embed(self.ids, self.table, self.x, factor=0.5)
        psk.psk_moe_route(self.x, self.router, self.crd, self.vals, ws=self.ws[0])
        psk.psk_moe_experts(self.x, self.crd, self.vals, self.w1, self.w3, self.w2, self.z, ws=self.ws[1])
        psk.psk_linear_i8(self.table, self.z, self.logits, ws=self.ws[2])
        psk.psk_embed_grad(self.ids, self.z, self.grad, factor=0.5, padding=7, ws=self.ws[3])

    def outputs(self):
        return [t.clone() for t in (self.x, self.z, self.logits, self.grad)]

    def check(self, what):
        """Each operator on what it was given."""
        cpu = [t.cpu() for t in (self.ids, self.codes, self.scales, self.x, self.z, self.logits, self.grad)]
        ids, codes, scales, x, z, logits, grad = cpu
        R.check(x, *R.embed(ids, codes, 0.5, torch.float16, scales), what + ": lookup")
        q, s = R.quantised(z)
        R.check(logits, *R.product(q, codes.long(), scales, s, None, torch.float16), what + ": logits")
        R.check(grad, *R.embed_grad(ids, z, self.vocab, 0.5, 7, torch.float32), what + ": gradient")


@pytest.mark.parametrize("n", [1, 5, 40, 300])
def test_a_run_of_them(n):
    m = Model(n, n)
    m.run()
    m.check("eager")


@pytest.mark.parametrize("n", [1, 9, 200])
def test_captured_and_replayed_with_new_tokens(n):
    m = Model(n, 20 + n)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        m.run()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.run()
    for i in range(4):
        m.ids.copy_(torch.randint(-1, m.vocab, (n,), generator=torch.Generator().manual_seed(i), dtype=torch.int32))
        m.run()
        want = m.outputs()
        for t in (m.x, m.z, m.logits, m.grad):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(m.outputs(), want)), i
        if i == 0:
            m.check("replayed")


def test_two_graphs_share_a_workspace():
    """Replayed one after the other on one stream, in either order."""
    a, b = Model(30, 1), Model(70, 2)
    for i in range(4):                                      # the larger of each pair serves both
        a.ws[i] = b.ws[i] = max(a.ws[i], b.ws[i], key=lambda t: t.numel())
    graphs = []
    for m in (a, b):
        m.run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            m.run()
        graphs.append(graph)
    want = [m.run() or m.outputs() for m in (a, b)]
    for order in ((0, 1, 1, 0), (1, 0, 0, 1)):
        for k in order:
            graphs[k].replay()
        torch.cuda.synchronize()
        for m, w in zip((a, b), want):
            assert all(torch.equal(x, y) for x, y in zip(m.outputs(), w))


def test_two_streams_at_once():
    """Calls with workspaces of their own, side by side, the stream given to the call."""
    models = [Model(257, 5), Model(33, 6)]
    want = [m.run() or m.outputs() for m in models]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in models]
    for _ in range(5):
        for m, s in zip(models, streams):
            psk.psk_embed(m.ids, m.table, m.x, factor=0.5, stream=s)
            psk.psk_linear_i8(m.table, m.z, m.logits, ws=m.ws[2], stream=s)
            psk.psk_embed_grad(m.ids, m.z, m.grad, factor=0.5, padding=7, stream=s)       # a workspace of the call's own
    torch.cuda.synchronize()
    for m, w in zip(models, want):
        assert all(torch.equal(x, y) for x, y in zip(m.outputs(), w))


def test_without_a_workspace_and_beside_other_work():
    m = Model(50, 9)
    m.run()
    want = m.outputs()
    m.logits.fill_(0)
    m.grad.fill_(1)
    psk.psk_linear_i8(m.table, m.z, m.logits)
    psk.psk_embed_grad(m.ids, m.z, m.grad, factor=0.5, padding=7)
    junk = [torch.full((1 << 20,), 0xff, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert all(torch.equal(x, y) for x, y in zip(m.outputs(), want)) and len(junk) == 4
