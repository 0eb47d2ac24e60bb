"""The vocabulary losses and the microscaled linear layer inside a CUDA graph, on two streams at
once, and mixed with the other kernels of the library that use tensor memory."""
import pytest

torch = pytest.importorskip("torch")

import paper_2403_06082_gb300 as fq  # noqa: E402
from fqgpu import DeviceLayer, activations, oracle_layer  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16 = torch.bfloat16


class Step:
    """A hidden state from a microscaled layer, its distillation loss, and both gradients."""

    def __init__(self, M, d, V, K, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.M, self.d, self.V, self.K = M, d, V, K
        self.x = torch.randn(M, d, generator=g, device=DEV).to(BF16)
        w1 = (torch.randn(d, d, generator=g, device=DEV) / d ** 0.5).to(BF16)
        self.q = fq.fq_mxfp_alloc(d, d)
        fq.fq_mxfp_quantize(w1, d, d, self.q)
        self.W = (torch.randn(V, d, generator=g, device=DEV) / d ** 0.5).to(BF16)
        self.index = torch.randint(-1, V, (M, K), generator=g, device=DEV).to(torch.int32)
        self.logit = torch.randn(M, K, generator=g, device=DEV)
        self.dloss = torch.randn(M, generator=g, device=DEV)
        self.h, self.dx = torch.empty_like(self.x), torch.empty_like(self.x)
        self.dW = torch.empty_like(self.W)
        self.loss, self.lse = torch.empty(M, device=DEV), torch.empty(M, device=DEV)
        self.n1 = fq.fq_mxfp_workspace_bytes(M, d, d)
        self.n2 = max(fq.fq_head_workspace_bytes(M, d, V, K),
                      fq.fq_head_grad_workspace_bytes(M, d, V, K))
        self.ws1 = torch.empty(self.n1, dtype=torch.uint8, device=DEV)
        self.ws2 = torch.empty(self.n2, dtype=torch.uint8, device=DEV)

    def run(self):
        fq.fq_mxfp_linear(self.x, self.M, self.d, self.q, self.h, self.ws1, self.n1)
        head = (self.h, self.M, self.d, self.W, self.V, self.index, self.logit, self.K, 2.0)
        fq.fq_distill(*head, self.loss, self.lse, self.ws2, self.n2)
        fq.fq_distill_grad(*head, self.lse, self.dloss, self.dx, self.dW, self.ws2, self.n2)

    def out(self):
        return [t.clone() for t in (self.h, self.loss, self.lse, self.dx, self.dW)]

    def clear(self):
        for t in (self.h, self.loss, self.lse, self.dx, self.dW):
            t.fill_(float("nan"))


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("M,d,V,K", [(1, 256, 1000, 3), (48, 512, 2003, 8), (300, 256, 5001, 16)])
def test_graph_replays_give_the_same_bits(M, d, V, K):
    s = Step(M, d, V, K, 1)
    s.run()
    torch.cuda.synchronize()
    want = s.out()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
        s.run()
    for _ in range(3):
        s.clear()
        graph.replay()
        torch.cuda.synchronize()
        assert _same(s.out(), want)
    # new inputs in the same buffers
    s.x.copy_(torch.randn_like(s.x))
    s.run()
    torch.cuda.synchronize()
    want = s.out()
    s.clear()
    graph.replay()
    torch.cuda.synchronize()
    assert _same(s.out(), want)


def test_two_streams_at_once():
    steps = [Step(200, 512, 4001, 8, 2), Step(31, 768, 3001, 4, 3)]
    want = []
    for s in steps:
        s.run()
        torch.cuda.synchronize()
        want.append(s.out())
        s.clear()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(20):
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                s.run()
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        assert _same(s.out(), w)
        assert fq.fq_check(s.ws1) == 0 and fq.fq_check(s.ws2) == 0


def test_mixed_with_the_frame_quantized_layer():
    """The layer's fused kernel before and after the operators on one stream, over and over: each
    starts while the one before it drains, and every result is what it is alone."""
    L = oracle_layer("single256", "single")
    D = DeviceLayer(L, BF16)
    X = activations("single256", "single", 16)
    ref = D.forward(X)
    x = torch.from_numpy(X).to(DEV, BF16)
    s = Step(16, 256, 1500, 4, 4)
    s.run()
    torch.cuda.synchronize()
    want = s.out()
    n = fq.fq_workspace_bytes(16, L.d_in, L.n_in, L.n_out, L.d_out, fq.FQ_BF16)
    ws = torch.zeros(n, dtype=torch.uint8, device=DEV)
    ys = []
    for _ in range(20):
        y = torch.empty(16, L.d_out, dtype=BF16, device=DEV)
        fq.fq_linear_forward(x, 16, L.d_in, D.T_in, D.C, D.T_out_t, L.d_out, None, y, ws, n)
        s.run()
        ys.append(y)
    torch.cuda.synchronize()
    assert _same(s.out(), want)
    for y in ys:
        assert (y.double().cpu().numpy() == ref).all()
