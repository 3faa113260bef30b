"""The token operators together with the compressed layers, as a training step uses them: embedding -> linear layer (compressed
activation) -> tied output layer -> loss with its gradient -> weight gradients -> AdamW, against the same step in 64 bits on the
CPU.  The layer's ranks are full, so that the compressed gradient equals the vanilla one; its tolerance is the one the
library's parity tests use, and everything behind it inherits that."""
import numpy as np
import pytest
import torch

from oracle import asi_oracle as O
from tests.gpu_util import TOL_F32

pytestmark = pytest.mark.gpu
B, N, D, V = 4, 6, 16, 40
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-6, weight_decay=0.01)


def setup(seed=0):
    g = np.random.default_rng(seed)
    # activations of full rank in every mode, well conditioned
    table = g.standard_normal((V, D)).astype(np.float32)
    W = (np.eye(D) + 0.2 * g.standard_normal((D, D))).astype(np.float32)
    ids = g.permutation(V)[: B * N].reshape(B, N)
    ids[3, 5] = ids[0, 0]                                            # one id twice
    targets = g.integers(0, V, B * N)
    targets[2] = -100
    U0 = [np.linalg.qr(g.standard_normal((d, d)))[0].astype(np.float32) for d in (B, N, D)]
    return table, W, ids, targets, U0


def plain_gradients(table, W, ids, targets, scale):
    """Loss and gradients of table (lookup and output layer) and W in 64 bits, and the layer's input."""
    t, w = (torch.tensor(x, dtype=torch.float64, requires_grad=True) for x in (table, W))
    x = scale * t[torch.from_numpy(ids)]
    h = x @ w.T
    logits = h.reshape(B * N, D) @ t.T
    y = torch.from_numpy(targets)
    lp = torch.log_softmax(logits, 1)
    live = y >= 0
    loss = -lp[live, y[live]].mean()
    loss.backward()
    return float(loss.detach()), t.grad.numpy(), w.grad.numpy(), x.detach().numpy()


def gpu_gradients(table, W, ids, targets, scale, U0):
    from paper_2505_05086_b200.runner import EmbeddingRunner, LayerRunner, LogprobRunner
    dev = "cuda:0"
    t, w = torch.from_numpy(table).to(dev), torch.from_numpy(W).to(dev)
    ids_d, y = torch.from_numpy(ids).to(dev), torch.from_numpy(targets).to(dev)
    emb = EmbeddingRunner(V, D, B * N, scale=scale)
    layer = LayerRunner("linear", (B, N, D), (B, N, D), D)
    head = LogprobRunner(B * N, V)
    x = torch.empty(B, N, D, device=dev)
    emb.forward(t, ids_d, x)
    layer.set_factors(U0)
    layer.compress(x)
    h = (x.double() @ w.double().T).reshape(B * N, D)
    logits = (h @ t.double().T).float()
    live = y >= 0
    weights = torch.where(live, -1.0 / live.sum(), 0.0).float()
    dlogits = torch.empty_like(logits)
    head.loss(logits, y, weights, None, dlogits)
    loss = float((weights * head.logp).sum())
    dh = (dlogits.double() @ t.double()).float().reshape(B, N, D)
    layer.wgrad(dh)
    assert layer.ok()
    dt = (dlogits.double().T @ h).float().contiguous()               # the output layer's gradient, and the lookup's on top
    dx = (dh.double() @ w.double()).float().contiguous()
    emb.wgrad(ids_d, dx, dt, accumulate=True)
    return loss, dt, layer.dW.view(D, D).clone()


def test_gradients_of_a_step():
    table, W, ids, targets, U0 = setup()
    loss, gt, gw, x = plain_gradients(table, W, ids, targets, 1.5)
    got, dt, dw = gpu_gradients(table, W, ids, targets, 1.5, U0)
    # every path is fp32 with sums of at most V terms: 64 u of the norms, u = 2^-24; the layer's by its own tolerance
    assert abs(got - loss) <= 64 * 2.0 ** -24 * (1 + abs(loss))
    assert O.rel_fro(dt.cpu().numpy(), gt) <= 64 * 2.0 ** -24 * 8
    assert O.rel_fro(dw.cpu().numpy(), gw) <= TOL_F32["dw"]


@pytest.mark.parametrize("bits8", [False, True])
def test_gradient_buffers_of_a_step_runner_feed_the_optimizer(bits8):
    """Two compressed layers behind the batched calls, and AdamW over their dW buffers, for three steps."""
    from paper_2505_05086_b200.runner import LayerRunner, StepRunner
    g = np.random.default_rng(1)
    shapes = [((4, 5, 12), (4, 5, 12), 10), ((4, 5, 10), (4, 5, 10), 7)]
    layers = [LayerRunner("linear", d, r, c) for d, r, c in shapes]
    for layer, (d, _, _) in zip(layers, shapes):
        layer.set_factors([np.linalg.qr(g.standard_normal((k, k)))[0] for k in d])
    step = StepRunner(layers)
    weights = [torch.randn(c, d[-1], device="cuda") for d, _, c in shapes]
    ref = [w.double().cpu().numpy() for w in weights]
    m, v = [np.zeros_like(w) for w in ref], [np.zeros_like(w) for w in ref]
    opt = step.optimizer(weights, bits8=bits8)
    for t in range(1, 4):
        acts = [g.standard_normal(d).astype(np.float32) for d, _, _ in shapes]
        dys = [g.standard_normal(d[:-1] + (c,)).astype(np.float32) for d, _, c in shapes]
        step.compress([layer.to_device(a) for layer, a in zip(layers, acts)])
        step.wgrad([layer.to_device(a) for layer, a in zip(layers, dys)])
        opt.step(**HYPER)
        for i, (a, dy) in enumerate(zip(acts, dys)):
            dw = np.einsum("bno,bnk->ok", dy.astype(np.float64), a.astype(np.float64))
            m[i] = HYPER["beta1"] * m[i] + (1 - HYPER["beta1"]) * dw
            v[i] = HYPER["beta2"] * v[i] + (1 - HYPER["beta2"]) * dw * dw
            up = HYPER["lr"] / (1 - HYPER["beta1"] ** t) * m[i] / (np.sqrt(v[i] / (1 - HYPER["beta2"] ** t)) + HYPER["eps"])
            ref[i] = ref[i] * (1 - HYPER["lr"] * HYPER["weight_decay"]) - up
    assert all(layer.ok() for layer in layers)
    for w, r in zip(weights, ref):
        off = np.abs(w.double().cpu().numpy() - r)
        if bits8:
            # each step's states carry a rounding of 2^-4 (m, sqrt(v)) on to the next: an update is off by at most about
            # 2^-4 of lr |m| / sqrt(v) <= lr, twice, for two of the three steps (and small second moments by their floor)
            assert np.linalg.norm(off) <= 2 * 2 * 2.0 ** -4 * HYPER["lr"] * np.sqrt(off.size) * 2
        else:
            # dW off by TOL_F32["dw"] of its norm; an update lr m / sqrt(v) moves by at most twice that relative, three times,
            # where an element is as large as the norm's mean; the norm of what is off stays below ten times that
            assert np.linalg.norm(off) <= 10 * 3 * 2 * TOL_F32["dw"] * HYPER["lr"] * np.sqrt(off.size)


@pytest.mark.parametrize("bits8", [False, True])
def test_a_whole_step_in_a_graph(bits8):
    """Loss, embedding gradient and AdamW captured and replayed: the same bits as the calls one by one."""
    from paper_2505_05086_b200.runner import AdamWRunner, EmbeddingRunner, LogprobRunner

    def world():
        g = torch.Generator(device="cuda").manual_seed(5)
        T, v, d = 300, 1000, 64
        s = dict(table=torch.randn(v, d, generator=g, device="cuda"), ids=torch.randint(0, v, (T,), generator=g, device="cuda"),
                 y=torch.randint(0, v, (T,), generator=g, device="cuda"), x=torch.empty(T, d, device="cuda"),
                 logits=torch.randn(T, v, generator=g, device="cuda"), w=torch.full((T,), -1 / T, device="cuda"),
                 dl=torch.empty(T, v, device="cuda"), dt=torch.empty(v, d, device="cuda"),
                 t=torch.ones(1, dtype=torch.int64, device="cuda"))
        s["emb"], s["head"] = EmbeddingRunner(v, d, T), LogprobRunner(T, v)
        s["opt"] = AdamWRunner([s["table"]], [s["dt"]], bits8=bits8)
        return s

    def go(s):
        s["emb"].forward(s["table"], s["ids"], s["x"])
        s["head"].loss(s["logits"], s["y"], s["w"], None, s["dl"])
        s["emb"].wgrad(s["ids"], s["x"], s["dt"])
        s["opt"].step(step=s["t"], **HYPER)
        s["t"] += 1

    a, b = world(), world()
    go(a), go(b)                                                     # (workspaces exist)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(b)
    for _ in range(4):
        go(a)
        graph.replay()
    torch.cuda.synchronize()
    for k in ("table", "x", "dl", "dt", "t"):
        assert torch.equal(a[k], b[k]), k
    assert torch.equal(a["opt"].exp_avg_sq[0].view(torch.uint8), b["opt"].exp_avg_sq[0].view(torch.uint8))
