"""The block operators' definitions in 64 bits, for their tests: dropout masks from the counter-based generator, block ends, and the output
layer with its loss."""
import numpy as np
import torch

from oracle.gaussian_stream import philox4x32_10

U32, U16 = 2.0 ** -24, 2.0 ** -8         # half a step of fp32 and of bf16, relative


def half_words(seed, stream, step, first, n):
    """Sixteen bits of each of the elements first .. first + n - 1."""
    g0, g1 = first // 8, (first + n + 7) // 8
    g = np.arange(g0, g1, dtype=np.uint64)
    low, full = np.uint64(0xFFFFFFFF), np.ones_like(g)
    ctr = np.stack([g & low, g >> np.uint64(32), full * np.uint64(stream), full * np.uint64(step & 0xFFFFFFFF)], 1).astype(np.uint32)
    key = np.array([seed & 0xFFFFFFFF, seed >> 32], dtype=np.uint32)
    words = np.asarray(philox4x32_10(ctr, np.broadcast_to(key, (len(g), 2)))).astype(np.uint32).reshape(len(g), 4)
    halves = np.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)
    return halves[first - 8 * g0:first - 8 * g0 + n]


def factors(p, seed, stream, step, n, first=0):
    """What dropout multiplies each element with."""
    k = int(np.floor(p * 65536 + 0.5))
    return torch.from_numpy(np.where(half_words(seed, stream, step, first, n) < k, 0.0, 65536 / (65536 - k)))


def norm(x, layer, w, b, eps):
    m = x.mean(1, keepdim=True) if layer else 0.0
    x = x - m
    x = x / (x.square().mean(1, keepdim=True) + eps).sqrt()
    x = x if w is None else x * w
    return x if b is None else x + b


def head(x, w, y, scale, ignore, dlogp=None, dent=None):
    """logp, entropy, lse and, for given weights, the logits' gradient G; also p and the bound S of the rows' |x| |w| sums."""
    x, w = x.double(), w.double()
    logits = scale * (x @ w.T)
    lse = torch.logsumexp(logits, 1)
    lp = logits - lse[:, None]
    p = lp.exp()
    ent = -torch.where(p > 0, p * lp, 0.0).sum(1)
    at = torch.arange(len(y), device=y.device)
    ok, live = (y >= 0) & (y < len(w)), y != ignore
    logp = torch.where(live, torch.where(ok, lp[at, y.clamp(0, len(w) - 1)], float("nan")), 0.0)
    out = dict(logp=logp, entropy=ent, lse=lse, p=p, S=scale * (x.abs() @ w.abs().T).amax(1))
    if dlogp is not None:
        a = torch.where(live, torch.where(ok, dlogp.double(), float("nan")), 0.0)[:, None]
        hot = torch.zeros_like(p)
        hot[at, y.clamp(0, len(w) - 1)] = ok.double()
        g, size = a * (hot - p), a.abs() * (hot + p)
        if dent is not None:
            b = torch.where(live, dent.double(), 0.0)[:, None]
            h = torch.where(p > 0, p * (lp + ent[:, None]), 0.0)
            g, size = g - b * h, size + b.abs() * p * (lp.abs() + ent[:, None])
        g = torch.where(live[:, None], scale * g, 0.0)
        out.update(G=g, size=scale * size, dx=g @ w, dw=g.T @ x)
    return out
