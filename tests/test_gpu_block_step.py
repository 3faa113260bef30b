"""Block ends, dropout and the output layer with its loss together with the compressed layers, as a training step uses them: embedding ->
norm -> linear layer (compressed activation) -> dropout, gate and residual sum, norm -> loss over the tied table -> gradients -> AdamW,
against the same step in 64 bits.  The layer's ranks are full, so that its compressed gradient equals the vanilla one."""
import numpy as np
import pytest
import torch

from oracle import asi_oracle as O
from tests.block_util import factors, norm
from tests.gpu_util import TOL_F32

pytestmark = pytest.mark.gpu
B, N, D, V = 4, 6, 16, 40
T, EPS = B * N, 1e-5
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-6, weight_decay=0.01)


def setup():
    g = torch.Generator(device="cuda").manual_seed(3)

    def normal(*s):
        return torch.randn(*s, generator=g, device="cuda")
    W = dict(table=normal(V, D), W=torch.eye(D, device="cuda") + 0.2 * normal(D, D), first=1 + 0.1 * normal(D), after=1 + 0.1 * normal(D),
             gate=0.5 + 0.1 * normal(1, D), last=1 + 0.1 * normal(D))
    ids = torch.randperm(V, generator=g, device="cuda")[:T]
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    y[2] = -100
    return W, ids, y


def plain(W, ids, y, step):
    """Loss and gradients in 64 bits."""
    p = {k: v.double().detach().requires_grad_(True) for k, v in W.items()}
    h = p["table"][ids]
    z = norm(h, False, p["first"], None, EPS) @ p["W"].T
    u = norm(z, False, p["after"], None, EPS) * p["gate"] * factors(0.2, 17, 1, step, T * D).view(T, D).cuda()
    x = norm(h + 1.5 * u, False, p["last"], None, EPS)
    logp = torch.log_softmax(x @ p["table"].T, 1)
    live = y >= 0
    loss = -logp[live, y[live]].mean()
    loss.backward()
    return float(loss.detach()), {k: v.grad for k, v in p.items()}


class Step:
    def __init__(self, W, ids, y):
        from paper_2505_05086_b200.runner import AdamWRunner, EmbeddingRunner, HeadRunner, LayerRunner, ResidualNormRunner
        self.W, self.ids, self.y = W, ids, y

        def buf(*s):
            return torch.zeros(*s, device="cuda")
        self.emb, self.layer, self.head = EmbeddingRunner(V, D, T), LayerRunner("linear", (B, N, D), (B, N, D), D), HeadRunner(T, V, D)
        self.begin = ResidualNormRunner(T, D, eps=EPS)
        self.end = ResidualNormRunner(T, D, norm_after=True, rows_per_gate=T, eps=EPS, branch_scale=1.5, dropout=0.2, seed=17, stream_id=1)
        g = np.random.default_rng(0)
        self.layer.set_factors([np.linalg.qr(g.standard_normal((d, d)))[0].astype(np.float32) for d in (B, N, D)])
        self.h0, self.h, self.x0, self.z, self.h2, self.x = (buf(T, D) for _ in range(6))
        self.g = {k: torch.zeros_like(v) for k, v in W.items()}
        self.dx, self.dz, self.dh, self.dx0, self.de = (buf(T, D) for _ in range(5))
        self.weights = torch.where(y >= 0, -1.0 / (y >= 0).sum(), 0.0).float()
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.g["W"] = self.layer.dW.view(D, D)
        self.names = list(W)
        self.opt = AdamWRunner([W[k] for k in self.names], [self.g[k] for k in self.names])

    def gradients(self):
        W, g = self.W, self.g
        self.emb.forward(W["table"], self.ids, self.h0)
        self.begin.forward(self.h0, None, self.h, self.x0, next=(W["first"], None))
        self.layer.compress(self.x0.view(B, N, D))
        torch.matmul(self.x0, W["W"].T, out=self.z)
        self.end.forward(self.z, self.h, self.h2, self.x, gate=W["gate"], after=(W["after"], None), next=(W["last"], None), step=self.step)
        self.head.loss(self.x, W["table"], self.y, self.weights, None, self.dx, g["table"])
        self.end.backward(self.z, self.h2, self.dx, None, self.dz, self.dh, gate=W["gate"], after=(W["after"], None), next=(W["last"], None),
                          dgate=g["gate"], dafter=(g["after"], None), dnext=(g["last"], None), step=self.step)
        self.layer.wgrad(self.dz.view(B, N, D))
        torch.matmul(self.dz, W["W"], out=self.dx0)
        self.begin.backward(self.h0, self.h, self.dx0, self.dh, self.de, None, next=(W["first"], None), dnext=(g["first"], None))
        self.emb.wgrad(self.ids, self.de, g["table"], accumulate=True)

    def go(self):
        self.gradients()
        self.step += 1
        self.opt.step(step=self.step, **HYPER)


def test_gradients_of_a_step():
    W, ids, y = setup()
    s = Step(W, ids, y)
    s.step.fill_(5)
    s.gradients()
    assert s.layer.ok() and s.head.device_status() == 0
    loss, want = plain(W, ids, y, 5)
    assert abs(float((s.weights * s.head.logp).sum()) - loss) <= 256 * 2.0 ** -24 * (1 + loss)
    for k, v in want.items():
        # fp32 all along with sums of at most V terms, and two products in torch's fp32: 1024 half steps of the norms; the layer's by its own tolerance
        tol = TOL_F32["dw"] if k == "W" else 1024 * 2.0 ** -24
        assert O.rel_fro(s.g[k].cpu().numpy(), v.cpu().numpy()) <= tol, k


def test_steps_in_a_graph_and_one_by_one():
    a, b = (Step(*(x if isinstance(x, torch.Tensor) else {k: v.clone() for k, v in x.items()} for x in setup())) for _ in range(2))
    for s in (a, b):
        s.go()
        s.layer.cur = 0                                               # (a graph goes on from the same factors each time)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.go()
    b.layer.cur = 0
    for _ in range(3):
        a.go()
        a.layer.cur = 0
        graph.replay()
    torch.cuda.synchronize()
    for k in a.names:
        assert torch.equal(a.W[k], b.W[k]) and torch.equal(a.g[k], b.g[k]), k
    assert torch.equal(a.head.logp, b.head.logp) and int(a.step) == 4
