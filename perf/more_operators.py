"""Operators of a transformer block and of its output layer, as measurable cases.

kind "dropout"  dropout from a counter-based generator (the mask is never stored), with or without a residual added
kind "branch"   what joins a block's branch to the residual stream: norm after the block, gate, dropout, scales and sum, and the
                norm before the next block
kind "bgrad"    its gradient, for branch, residual stream, gate and the norms' weights
kind "score"    log probabilities of given tokens straight from the last hidden states and the output layer's weight
kind "head"     the same with the gradients of hidden states and weight in one call; the logits are never kept

Hidden states are Gaussian, as a norm leaves them; output rows have logits of spread 2.5 and most tokens lean to their target.
"""
import math

import numpy as np
import torch

own = False

IGNORE = -100
EPS = 1e-5
DT = {True: torch.bfloat16, False: torch.float32}
MOST_DROP, MOST_BRANCH, MOST_HEAD, MOST_LOGITS, MOST_WEIGHT = 16e6, 12e6, 2.6e11, 1.3e8, 6.5e7


def listed():
    return [
        # four sequences of a policy that samples with dropout on: nothing but latency
        dict(name="dropout-tokens", kind="dropout", n=4 * 2048, bf16=True, p=0.1, res=False),
        # a branch of 8 sequences of 512 tokens, added to its residual stream
        dict(name="dropout-4096", kind="dropout", n=4096 * 2048, bf16=True, p=0.1, res=True),
        # a ragged batch in fp32, odd sizes
        dict(name="dropout-ragged", kind="dropout", n=1001 * 771, bf16=False, p=0.35, res=False),
        # four tokens through a block's end
        dict(name="branch-tokens", kind="branch", T=4, D=2048, bf16=True, bf16_res=True, layer=False, after=True, per_gate=0, p=0.0),
        # norms before and after a block, learned gate, 8 sequences of 512 tokens, residual stream in bf16
        dict(name="branch-4096", kind="branch", T=4096, D=2048, bf16=True, bf16_res=True, layer=False, after=True, per_gate=0, p=0.0),
        # the gradient of the same
        dict(name="bgrad-4096", kind="bgrad", T=4096, D=2048, bf16=True, bf16_res=True, layer=False, after=True, per_gate=0, p=0.0),
        # images: 32 of 197 tokens, layer norms, a gate for each image, dropout, residual stream in fp32
        dict(name="bgrad-images", kind="bgrad", T=32 * 197, D=768, bf16=True, bf16_res=False, layer=True, after=False, per_gate=197, p=0.1),
        # odd sizes in fp32 throughout, norms on both sides, no dropout
        dict(name="bgrad-ragged", kind="bgrad", T=1001, D=771, bf16=False, bf16_res=False, layer=True, after=True, per_gate=0, p=0.0),
        # scoring 8 sequences of 512 tokens
        dict(name="score-4096", kind="score", T=4096, V=32000, D=2048, bf16=True, scale=1.0),
        # fine-tuning on them: loss and both gradients
        dict(name="head-4096", kind="head", T=4096, V=32000, D=2048, bf16=True, bf16_dw=True, add=False, ent=False, scale=1.0),
        # a few tokens of a small model, the weight's gradient added to a tied embedding's in fp32
        dict(name="head-few", kind="head", T=9, V=50257, D=768, bf16=True, bf16_dw=False, add=True, ent=False, scale=1.0),
        # a ragged batch in fp32, odd sizes, an entropy bonus and a temperature
        dict(name="head-ragged", kind="head", T=1001, V=30011, D=771, bf16=False, bf16_dw=False, add=False, ent=True, scale=0.7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["dropout", "branch", "bgrad", "score", "head", "head"])
    b = rng.random() < 0.6
    if kind == "dropout":
        return dict(kind=kind, n=_log(rng, 500, MOST_DROP), bf16=b, p=round(rng.uniform(0.01, 0.6), 3), res=rng.random() < 0.5)
    if kind in ("branch", "bgrad"):
        D = _log(rng, 33, 8192)
        T = _log(rng, 1, min(16384, MOST_BRANCH / D))
        return dict(kind=kind, T=T, D=D, bf16=b, bf16_res=b and rng.random() < 0.5, layer=rng.random() < 0.5, after=rng.random() < 0.6,
                    per_gate=rng.choice([0, 0, -1, 1, max(1, T // 7)]), p=rng.choice([0.0, 0.0, 0.1]))
    V, D = _log(rng, 300, 130000), _log(rng, 65, 4500)
    V = max(300, min(V, int(MOST_WEIGHT / D)))
    T = _log(rng, 1, max(2, min(8192, MOST_LOGITS / V, MOST_HEAD / V / D)))
    c = dict(kind=kind, T=T, V=V, D=D, bf16=b, scale=rng.choice([1.0, 0.7, 1.25]))
    if kind == "head":
        c.update(bf16_dw=b and rng.random() < 0.6, add=rng.random() < 0.4, ent=rng.random() < 0.3)
    return c


# ---- inputs --------------------------------------------------------------------------------------

def _gates(case):
    """Rows of the gate, and tokens that share one."""
    per = case["per_gate"] or case["T"]
    return (0, 1) if per < 0 else (-(-case["T"] // per), per)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, s = case["kind"], dict(case=case, seed=seed * 0x9E3779B97F4A7C15 % (1 << 64), step=seed % 1000)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    if kind == "dropout":
        dt = DT[case["bf16"]]
        s["x"], s["out"] = normal(case["n"]).to(dt), torch.zeros(case["n"], device="cuda", dtype=dt)
        s["res"] = normal(case["n"]).to(dt) if case["res"] else None
        if own:
            from paper_2505_05086_b200.runner import DropoutRunner
            s["op"] = DropoutRunner(case["p"], s["seed"], stream_id=3, bf16=case["bf16"])
        return s
    if kind in ("branch", "bgrad"):
        T, D, dt, rt = case["T"], case["D"], DT[case["bf16"]], DT[case["bf16_res"]]
        rows, per = _gates(case)
        s["y"] = (0.7 * normal(T, D) + 0.1 * normal(D)).to(dt)
        s["gate"] = 0.5 + 0.2 * normal(rows, D) if rows else None
        s["aw"], s["ab"] = (1 + 0.1 * normal(D), 0.1 * normal(D) if case["layer"] else None) if case["after"] else (None, None)
        s["nw"], s["nb"] = 1 + 0.1 * normal(D), 0.1 * normal(D) if case["layer"] else None
        s["scales"] = (0.9, 1.2)                       # of the residual stream and of the branch
        h = 2 * normal(T, D).to(rt)
        if kind == "branch":
            s.update(h=h, h_out=torch.zeros(T, D, device="cuda", dtype=rt), x=torch.zeros(T, D, device="cuda", dtype=dt))
        else:                                          # what the forward pass left, and the gradients that come back
            s["h_out"] = h
            s["stats"] = torch.cat([_row_stats(s["y"], case["layer"]) if case["after"] else torch.zeros(T, 2, device="cuda"),
                                    _row_stats(h, case["layer"])], 1)
            s["dx"], s["dh_out"] = (0.1 * normal(T, D)).to(dt), (0.1 * normal(T, D)).to(rt)
            s["dy"], s["dh"] = torch.zeros(T, D, device="cuda", dtype=dt), torch.zeros(T, D, device="cuda", dtype=rt)
            for k in ("gate", "aw", "ab", "nw", "nb"):
                s["d" + k] = None if s[k] is None else torch.zeros_like(s[k])
        if own:
            from paper_2505_05086_b200.runner import ResidualNormRunner
            s["op"] = ResidualNormRunner(T, D, bf16=case["bf16"], bf16_residual=case["bf16_res"], norm="layer" if case["layer"] else "rms",
                                         norm_after=case["after"], rows_per_gate=per if rows else 0, eps=EPS, res_scale=s["scales"][0],
                                         branch_scale=s["scales"][1], dropout=case["p"], seed=s["seed"], stream_id=3)
            if kind == "bgrad":
                s["op"].stats.copy_(s["stats"])
        return s
    T, V, D, dt = case["T"], case["V"], case["D"], DT[case["bf16"]]
    s["w"] = (normal(V, D) * (2.5 / math.sqrt(D))).to(dt)
    s["y"] = torch.randint(0, V, (T,), generator=g, device="cuda")
    up = torch.rand(T, 1, generator=g, device="cuda")
    s["x"] = (normal(T, D) + torch.where(up < 0.7, 1.4 * up, 0.0) * s["w"][s["y"]].float()).to(dt)
    if kind == "head":
        s["y"][torch.rand(T, generator=g, device="cuda") < 0.1] = IGNORE
        s["dlogp"] = (torch.randn(T, generator=g, device="cuda") if case["ent"] else -torch.ones(T, device="cuda")) / T
        s["dent"] = 0.01 * torch.rand(T, generator=g, device="cuda") / T if case["ent"] else None
        s["dx"] = torch.zeros(T, D, device="cuda", dtype=dt)
        s["dw"] = (normal(V, D) / (4 * T) if case["add"] else torch.zeros(V, D, device="cuda")).to(DT[case["bf16_dw"]])
    if own:
        from paper_2505_05086_b200.runner import HeadRunner
        s["op"] = HeadRunner(T, V, D, bf16=case["bf16"], bf16_dw=case.get("bf16_dw", False), scale=case["scale"], ignore_index=IGNORE,
                             grad=kind == "head")
    return s


def _row_stats(x, layer):
    """Mean (0 where the norm has none) and reciprocal deviation of each row."""
    x = x.double()
    m = x.mean(1, keepdim=True) if layer else torch.zeros(len(x), 1, device="cuda", dtype=torch.float64)
    return torch.cat([m, 1 / torch.sqrt((x - m).square().mean(1, keepdim=True) + EPS)], 1).float()


# ---- the operators in their plain form --------------------------------------------------------------

def _plain_rounds(c0, c1, c2, c3, k0, k1, left):
    """Philox4x32 on 64-bit integers that hold 32-bit words."""
    if not left:
        return torch.stack([c0, c1, c2, c3], 1)
    a, b, low = c0 * 0xD2511F53, c2 * 0xCD9E8D57, 0xFFFFFFFF
    return _plain_rounds((b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low,
                         (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low, left - 1)


def _plain_keep(s, n):
    """Which of n elements stay, and what they are multiplied with: element e by the (e mod 8)-th sixteen bits of group e div 8."""
    drop = math.floor(s["case"]["p"] * 65536 + 0.5)
    group = torch.arange(-(-n // 8), device="cuda")
    same = torch.zeros_like(group)
    w = _plain_rounds(group & 0xFFFFFFFF, group >> 32, same + 3, same + s["step"], s["seed"] & 0xFFFFFFFF, s["seed"] >> 32, 10)
    half = torch.stack([w & 0xFFFF, w >> 16], 2).view(-1)[:n]
    return half >= drop, 65536 / (65536 - drop)


def _plain_norm(x, stats, w, b):
    """(x - mean) / deviation, and that with weight and bias."""
    n = (x - stats[:, :1]) * stats[:, 1:]
    y = n if w is None else n * w
    return n, y if b is None else y + b


def _plain_stats(x, layer):
    m = x.mean(1, keepdim=True) if layer else torch.zeros_like(x[:, :1])
    return torch.cat([m, torch.rsqrt((x - m).square().mean(1, keepdim=True) + EPS)], 1)


def _plain_gate(s):
    """The gate of each row."""
    rows, per = _gates(s["case"])
    return s["gate"][torch.arange(s["case"]["T"], device="cuda") // per] if rows else 1.0


def _plain_branch(s):
    case = s["case"]
    y = s["y"].float()
    sa = torch.zeros(case["T"], 2, device="cuda")
    if case["after"]:
        sa = _plain_stats(y, case["layer"])
        y = _plain_norm(y, sa, s["aw"], s["ab"])[1]
    u = y * _plain_gate(s)
    if case["p"]:
        keep, more = _plain_keep(s, u.numel())
        u = torch.where(keep.view(u.shape), u * more, 0.0)
    s["h_out"].copy_(s["h"].float() * s["scales"][0] + u * s["scales"][1])
    h = s["h_out"].float()                             # the next norm reads what is stored
    sn = _plain_stats(h, case["layer"])
    s["x"].copy_(_plain_norm(h, sn, s["nw"], s["nb"])[1])
    return dict(h_out=s["h_out"], x=s["x"], stats=torch.cat([sa, sn], 1))


def _plain_norm_grad(d, n, deviation, w, layer):
    """Gradient of the norm's input from that of its output."""
    d = d if w is None else d * w
    out = d - n * (d * n).mean(1, keepdim=True)
    return (out - d.mean(1, keepdim=True) if layer else out) * deviation


def _plain_bgrad(s):
    case, layer = s["case"], s["case"]["layer"]
    dx, h = s["dx"].float(), s["h_out"].float()
    n, _ = _plain_norm(h, s["stats"][:, 2:], None, None)
    if s["nb"] is not None:
        s["dnb"].copy_(dx.sum(0))
    s["dnw"].copy_((dx * n).sum(0))
    d = s["dh_out"].float() + _plain_norm_grad(dx, n, s["stats"][:, 3:], s["nw"], layer)
    s["dh"].copy_(d * s["scales"][0])
    du = d * s["scales"][1]
    if case["p"]:
        keep, more = _plain_keep(s, du.numel())
        du = torch.where(keep.view(du.shape), du * more, 0.0)
    y = s["y"].float()
    n, z = _plain_norm(y, s["stats"][:, :2], s["aw"], s["ab"]) if case["after"] else (y, y)
    rows, per = _gates(case)
    if rows:
        s["dgate"].zero_().index_add_(0, torch.arange(case["T"], device="cuda") // per, du * z)
    dz = du * _plain_gate(s)
    if case["after"]:
        s["daw"].copy_((dz * n).sum(0))
        if s["ab"] is not None:
            s["dab"].copy_(dz.sum(0))
        dz = _plain_norm_grad(dz, n, s["stats"][:, 1:2], s["aw"], layer)
    s["dy"].copy_(dz)


def _plain_head(s):
    """Differences from each row's largest logit, log of the sum of their exponentials, and the outputs of the forward pass."""
    x = (s["x"].float() @ s["w"].float().T).mul_(s["case"]["scale"])
    m = x.amax(1, keepdim=True)
    x.sub_(m)
    e = torch.exp(x)
    z = e.sum(1, keepdim=True)
    logz = torch.log(z)
    ent = logz[:, 0] - torch.where(e > 0, e * x, 0.0).sum(1) / z[:, 0]
    here = s["y"] != IGNORE
    logp = torch.where(here, (x.gather(1, s["y"].clamp(min=0)[:, None]) - logz)[:, 0], 0.0)
    return x, logz, here, dict(logp=logp, entropy=ent, lse=(m + logz)[:, 0])


def _plain_head_grad(s, d, logz, here, ent):
    lp = d - logz
    p = torch.exp(lp)
    w = torch.where(here, s["dlogp"], 0.0)[:, None]
    g = -w * p
    g.scatter_add_(1, s["y"].clamp(min=0)[:, None], w)
    if s["dent"] is not None:
        g = g - torch.where(here, s["dent"], 0.0)[:, None] * torch.where(p > 0, p * (lp + ent[:, None]), 0.0)
    g = g * s["case"]["scale"]
    s["dx"].copy_(g @ s["w"].float())
    dw = g.T @ s["x"].float()
    s["dw"].copy_(s["dw"].float() + dw if s["case"]["add"] else dw)


def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if kind == "dropout":
        if own:
            s["op"].forward(s["x"], s["out"], step=s["step"], residual=s["res"])
        else:
            keep, more = _plain_keep(s, case["n"])
            u = torch.where(keep, s["x"].float() * more, 0.0)
            s["out"].copy_(u if s["res"] is None else u + s["res"].float())
        return dict(out=s["out"])
    if kind == "branch":
        if own:
            s["op"].forward(s["y"], s["h"], s["h_out"], s["x"], gate=s["gate"], after=(s["aw"], s["ab"]), next=(s["nw"], s["nb"]),
                            step=s["step"])
            return dict(h_out=s["h_out"], x=s["x"], stats=s["op"].stats)
        return _plain_branch(s)
    if kind == "bgrad":
        if own:
            s["op"].backward(s["y"], s["h_out"], s["dx"], s["dh_out"], s["dy"], s["dh"], gate=s["gate"], after=(s["aw"], s["ab"]),
                             next=(s["nw"], s["nb"]), dgate=s["dgate"], dafter=(s["daw"], s["dab"]), dnext=(s["dnw"], s["dnb"]),
                             step=s["step"])
        else:
            _plain_bgrad(s)
        return {k: s[k] for k in ("dy", "dh", "dgate", "daw", "dab", "dnw", "dnb") if s[k] is not None}
    if kind == "score":
        if own:
            s["op"].forward(s["x"], s["w"], s["y"])
            return dict(logp=s["op"].logp, entropy=s["op"].entropy, lse=s["op"].lse)
        return _plain_head(s)[3]
    if own:
        s["op"].loss(s["x"], s["w"], s["y"], s["dlogp"], s["dent"], s["dx"], s["dw"], accumulate=case["add"])
        out = dict(logp=s["op"].logp, entropy=s["op"].entropy, lse=s["op"].lse)
    else:
        d, logz, here, out = _plain_head(s)
        _plain_head_grad(s, d, logz, here, out["entropy"])
    return dict(out, dx=s["dx"], dw=s["dw"])


# ---- what a pass cannot do without ------------------------------------------------------------------

def work(case):
    kind, e = case["kind"], 2 if case["bf16"] else 4
    if kind == "dropout":
        return dict(bytes=case["n"] * e * (3 if case["res"] else 2), flops=2.0 * case["n"])
    if kind in ("branch", "bgrad"):
        T, D, r = case["T"], case["D"], 2 if case["bf16_res"] else 4
        rows = _gates(case)[0]
        weights = 4 * D * (rows + (1 + case["layer"]) * (1 + case["after"]))
        if kind == "branch":
            return dict(bytes=T * D * 2 * (e + r) + 16 * T + weights, flops=16.0 * T * D)
        return dict(bytes=T * D * 3 * (e + r) + 16 * T + 2 * weights, flops=32.0 * T * D)
    T, V, D = case["T"], case["V"], case["D"]
    if kind == "score":
        return dict(bytes=(T + V) * D * e + 20 * T, flops=2.0 * T * V * D)
    d = 2 if case["bf16_dw"] else 4
    return dict(bytes=(2 * T + V) * D * e + V * D * d * (1 + case["add"]) + 28 * T, flops=6.0 * T * V * D)


# ---- the definitions in 64 bits -----------------------------------------------------------------------

def _words(seed, step, groups):
    """Philox4x32-10 of the counters (group, 3, step) in unsigned NumPy words, four a group."""
    u = np.uint64
    low, c = u(0xFFFFFFFF), np.zeros((4, groups), dtype=np.uint64)
    c[0], c[2], c[3] = np.arange(groups, dtype=np.uint64), 3, step
    key = [u(seed % (1 << 32)), u(seed >> 32)]
    for _ in range(10):
        p, q = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = np.stack([(q >> u(32)) ^ c[1] ^ key[0], q & low, (p >> u(32)) ^ c[3] ^ key[1], p & low])
        key = [(key[0] + u(0x9E3779B9)) & low, (key[1] + u(0xBB67AE85)) & low]
    return c.T.astype(np.uint32)


def _kept(s, n):
    """1 / (1 - p) where an element stays, 0 where it is dropped."""
    drop = round(s["case"]["p"] * 65536)
    half = np.ascontiguousarray(_words(s["seed"], s["step"], (n + 7) // 8)).view(np.uint16).reshape(-1)[:n]     # (low half first)
    return torch.from_numpy(np.where(half < drop, 0.0, 1 / (1 - drop / 65536))).cuda()


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "dropout":
        out = s["x"].double() * _kept(s, case["n"])
        return dict(out=out + s["res"].double() if case["res"] else out)
    if kind in ("branch", "bgrad"):
        T, D = case["T"], case["D"]
        f = {k: s[k].double() for k in ("y", "gate", "aw", "ab", "nw", "nb") if s.get(k) is not None}
        rows, per = _gates(case)

        def norm(x, w, b):
            if case["layer"]:
                return torch.nn.functional.layer_norm(x, (D,), w, b, EPS)
            return x / (x.pow(2).mean(1, keepdim=True) + EPS).sqrt() * w

        def stats(x):
            m = x.mean(1) if case["layer"] else torch.zeros(T, device="cuda", dtype=torch.float64)
            return torch.stack([m, (x.pow(2).mean(1) - m * m + EPS) ** -0.5], 1)
        mask = _kept(s, T * D).view(T, D) if case["p"] else 1.0

        def branch(y, gate, aw, ab):
            z = norm(y, aw, ab) if case["after"] else y
            return (torch.repeat_interleave(gate, per, 0)[:T] * z if rows else z) * mask * s["scales"][1]
        if kind == "branch":
            u = branch(f["y"], f.get("gate"), f.get("aw"), f.get("ab"))
            h = s["h"].double() * s["scales"][0] + u
            stored = h.to(s["h_out"].dtype).double()
            st = stats(f["y"]) if case["after"] else torch.zeros(T, 2, device="cuda", dtype=torch.float64)
            return dict(h_out=h, x=norm(stored, f["nw"], f.get("nb")), stats=torch.cat([st, stats(stored)], 1))
        for v in f.values():
            v.requires_grad_(True)
        h = s["h_out"].double().requires_grad_(True)
        up = torch.autograd.grad((norm(h, f["nw"], f.get("nb")) * s["dx"].double()).sum(), [h] + [f[k] for k in ("nw", "nb") if k in f])
        d = s["dh_out"].double() + up[0]
        out = dict(zip(("dnw", "dnb"), up[1:]), dh=d * s["scales"][0])
        names = [k for k in ("y", "gate", "aw", "ab") if k in f]
        down = torch.autograd.grad((branch(f["y"], f.get("gate"), f.get("aw"), f.get("ab")) * d).sum(), [f[k] for k in names])
        return dict(out, **{"d" + k: v for k, v in zip(names, down)})
    out, dw, w = {}, 0.0, s["w"].double()
    for r in range(0, case["T"], 512):
        x, y = s["x"][r:r + 512].double(), s["y"][r:r + 512]
        lp = torch.log_softmax(x @ w.T * case["scale"], 1)
        p = lp.exp()
        some, at = y >= 0, torch.arange(len(y), device="cuda")
        ent = -torch.xlogy(p, p).sum(1)
        first = x @ w[0] * case["scale"]
        part = dict(logp=torch.where(some, lp[at, y.clamp(min=0)], 0.0), entropy=ent, lse=first - lp[:, 0])
        if kind == "head":
            a = s["dlogp"][r:r + 512].double() * some
            gr = -a[:, None] * p
            gr[at, y.clamp(min=0)] += a
            if s["dent"] is not None:
                gr -= (s["dent"][r:r + 512].double() * some)[:, None] * (torch.xlogy(p, p) + p * ent[:, None])
            gr *= case["scale"]
            part["dx"], dw = gr @ w, dw + gr.T @ x
        for k, v in part.items():
            out.setdefault(k, []).append(v)
    out = {k: torch.cat(v) for k, v in out.items()}
    if kind == "head":
        out["dw"] = s["dw"].double() + dw if case["add"] else dw
    return out
