"""The operators around the compressed layers of a language model's training step, as measurable cases.

kind "logprob"   log probabilities of given tokens, entropy and top alternatives from logits (forward only)
kind "grad"      their gradient with respect to the logits, for weights that come after the forward pass
kind "loss"      both in one pass, for weights that are known before it
kind "embed"     embedding lookup with scaling
kind "wgrad"     the embedding's weight gradient, overwritten or added to a gradient that is there
kind "adamw"     one AdamW step over many tensors, states in 32 or 8 bits

Logits are Gaussian with the given token raised in most rows, a few columns are masked with -inf as unused entries of
a vocabulary are; token ids fall off as words do (the r-th most frequent one with probability about 1 / r).
"""
import math

import numpy as np
import torch

own = False

IGNORE = -100
BLOCK = 256                      # elements that share a scale in the 8-bit states
HYPER = dict(lr=2e-5, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)
MOST_LOGITS, MOST_EMBED, MOST_ADAMW = 270e6, 300e6, 30e6
DT = {True: torch.bfloat16, False: torch.float32}


def listed():
    return [
        # four sequences being sampled: log probability of the chosen token, 20 alternatives; nothing but latency
        dict(name="logprob-decode", kind="logprob", T=4, V=32000, pad=0, bf16=True, k=20, scale=1.25),
        # scoring a batch of 8 sequences of 512 tokens, five alternatives each
        dict(name="logprob-score", kind="logprob", T=4096, V=32000, pad=0, bf16=True, k=5, scale=1.0),
        # a large odd vocabulary in fp32, rows padded to a multiple of something else, a short batch
        dict(name="logprob-wide", kind="logprob", T=257, V=131073, pad=7, bf16=False, k=1, scale=1.0),
        # policy gradient with an entropy bonus: weights known only after the forward pass
        dict(name="grad-4096", kind="grad", T=4096, V=32000, pad=0, bf16=True, ent=True, scale=1.0),
        # fine-tuning on the same batch: cross entropy and its gradient in one pass
        dict(name="loss-4096", kind="loss", T=4096, V=32000, pad=0, bf16=True, ent=False, scale=1.0),
        # a ragged last batch in fp32, odd vocabulary, entropy bonus, a temperature
        dict(name="loss-ragged", kind="loss", T=1001, V=50257, pad=0, bf16=False, ent=True, scale=0.7),
        # the lookup for the same batch, fp32 weights to bf16 activations
        dict(name="embed-4096", kind="embed", T=4096, V=32000, D=2048, bf16=True, bf16_table=False, scale=45.25),
        # its weight gradient, every row of the table written
        dict(name="wgrad-4096", kind="wgrad", T=4096, V=32000, D=2048, bf16=True, add=False, scale=45.25),
        # a tied table: added to the head's gradient; fp32, odd sizes
        dict(name="wgrad-tied", kind="wgrad", T=9973, V=50257, D=770, bf16=False, add=True, scale=1.0),
        # the projections of a block with fp32 weights and states and a bf16 copy for the next forward pass
        dict(name="adamw-block", kind="adamw", sizes="4194304,11534336,11534336", bits8=False, p_bf16=False,
             g_bf16=False, copy=True),
        # the same with 8-bit states: weights and gradients in bf16
        dict(name="adamw8-block", kind="adamw", sizes="4194304,11534336,11534336", bits8=True, p_bf16=True,
             g_bf16=True, copy=False),
        # the last layers of an image classifier with all their small tensors, 8-bit states, fp32 weights
        dict(name="adamw8-convs", kind="adamw", sizes=",".join(["36864,64,64"] * 6 + ["73728,128,128"] + ["147456,128,128"] * 7
             + ["589824,256,256"] * 5 + ["2359296,512,512", "512000,1000"]), bits8=True, p_bf16=False, g_bf16=False, copy=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logprob", "grad", "loss", "embed", "wgrad", "adamw"])
    b = rng.random() < 0.6
    if kind in ("logprob", "grad", "loss"):
        V = _log(rng, 300, 160000)
        T = _log(rng, 1, max(2, min(8192, MOST_LOGITS / (V * (2 if b else 4)))))
        c = dict(kind=kind, T=T, V=V, pad=rng.choice([0, 0, 1, 8, 63]), bf16=b, scale=rng.choice([1.0, 0.7, 1.25]))
        if kind == "logprob":
            return dict(c, k=rng.choice([0, 1, 5, 20, 32]))
        return dict(c, ent=rng.random() < 0.5)
    if kind in ("embed", "wgrad"):
        D = _log(rng, 33, 6000)
        V = _log(rng, 200, min(160000, MOST_EMBED / (D * 4)))
        T = _log(rng, 1, max(2, min(32768, MOST_EMBED / (D * 6))))
        c = dict(kind=kind, T=T, V=V, D=D, bf16=b, scale=rng.choice([1.0, 45.25]))
        return dict(c, bf16_table=rng.random() < 0.5) if kind == "embed" else dict(c, add=rng.random() < 0.5)
    left, sizes = _log(rng, 1000, MOST_ADAMW), []
    for _ in range(_log(rng, 1, 60)):
        sizes.append(_log(rng, 1, max(2, left)))
        left = max(1, left - sizes[-1])
    return dict(kind=kind, sizes=",".join(map(str, sizes)), bits8=rng.random() < 0.6, p_bf16=rng.random() < 0.4,
                g_bf16=b, copy=rng.random() < 0.3)


# ---- inputs --------------------------------------------------------------------------------------

def _ids(T, V, g):
    """Ids whose frequency falls off as 1 / rank."""
    rank = torch.exp(torch.rand(T, generator=g, device="cuda", dtype=torch.float64) * math.log(V + 1.0)).long() - 1
    return torch.randperm(V, generator=g, device="cuda")[rank.clamp_(0, V - 1)]


def _distinct(T, V):
    r = np.arange(1, V + 1, dtype=np.float64)
    p = np.log1p(1.0 / r) / math.log(V + 1.0)
    return float(np.sum(-np.expm1(T * np.log1p(-np.minimum(p, 1 - 1e-15)))))


def _spans(case):
    """[(first element, elements)] of the tensors in their flat buffers, each on a block of its own, and the whole."""
    at, out = 0, []
    for n in map(int, case["sizes"].split(",")):
        out.append((at, n))
        at += -(-n // BLOCK) * BLOCK
    return out, at


def _adamw_inputs(case, g):
    spans, n = _spans(case)
    on = torch.zeros(n, device="cuda")
    for at, k in spans:
        on[at:at + k] = 1

    def normal():
        return torch.randn(n, generator=g, device="cuda") * on
    # every tensor's gradients have a size of their own, spread over its elements
    spread = torch.exp(1.5 * normal()) * on
    s = dict(p=(0.02 * normal()).to(DT[case["p_bf16"]]), g=(1e-4 * spread * normal()).to(DT[case["g_bf16"]]), t=100)
    m, r = 3e-5 * spread * normal(), 1e-4 * spread * (0.5 + normal().abs()) * on
    if case["bits8"]:
        s["m"], s["m_exp"] = _to8(m, False)
        s["v"], s["v_exp"] = _to8(r, True)
    else:
        s["m"], s["v"] = m, r * r
    s["copy"] = torch.zeros(n, device="cuda", dtype=torch.bfloat16) if case["copy"] else None
    s["spans"] = spans
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, s = case["kind"], dict(case=case)
    if kind in ("logprob", "grad", "loss"):
        T, V, dt = case["T"], case["V"], DT[case["bf16"]]
        full = torch.randn(T, V + case["pad"], generator=g, device="cuda").mul_(2.5).to(dt)
        y = torch.randint(0, V - 8, (T,), generator=g, device="cuda")
        up = torch.rand(T, generator=g, device="cuda")
        rows = torch.arange(T, device="cuda")
        full[rows, y] += (9.0 * (up < 0.7) * up).to(dt)
        full[:, V - 8:V] = float("-inf")
        s["logits"], s["targets"] = full[:, :V], y
        if kind != "logprob":
            y[torch.rand(T, generator=g, device="cuda") < 0.1] = IGNORE
            w = torch.randn(T, generator=g, device="cuda") if case["ent"] else -torch.ones(T, device="cuda")
            s["dlogp"] = w / T
            s["dent"] = 0.01 * torch.rand(T, generator=g, device="cuda") / T if case["ent"] else None
            s["dlogits"] = torch.zeros(T, V + case["pad"], device="cuda", dtype=dt)[:, :V]
        if kind == "grad":         # what the forward pass left
            s["lse"], s["ent"] = _stats64(s["logits"], case["scale"])
        if own:
            from paper_2505_05086_b200.runner import LogprobRunner
            s["op"] = LogprobRunner(T, V, bf16=case["bf16"], scale=case["scale"], ignore_index=IGNORE, top_k=case.get("k", 0))
            if kind == "grad":
                s["op"].lse.copy_(s["lse"])
                s["op"].entropy.copy_(s["ent"])
    elif kind in ("embed", "wgrad"):
        T, V, D = case["T"], case["V"], case["D"]
        s["ids"] = _ids(T, V, g)
        if kind == "embed":
            s["table"] = (0.02 * torch.randn(V, D, generator=g, device="cuda")).to(DT[case["bf16_table"]])
            s["out"] = torch.zeros(T, D, device="cuda", dtype=DT[case["bf16"]])
        else:
            s["pad"] = int(s["ids"][0])
            s["ids"][torch.rand(T, generator=g, device="cuda") < 0.1] = s["pad"]
            s["dout"] = (torch.randn(T, D, generator=g, device="cuda") / T).to(DT[case["bf16"]])
            s["dw"] = torch.randn(V, D, generator=g, device="cuda") / T if case["add"] else torch.zeros(V, D, device="cuda")
        if own:
            from paper_2505_05086_b200.runner import EmbeddingRunner
            s["op"] = EmbeddingRunner(V, D, T, bf16=case["bf16"], bf16_table=case.get("bf16_table", False),
                                      scale=case["scale"], padding_idx=s.get("pad"))
    else:
        s.update(_adamw_inputs(case, g))
        if own:
            from paper_2505_05086_b200.runner import AdamWRunner

            def views(x, per=1):
                return None if x is None else [x[at // per:at // per + -(-n // per)] for at, n in s["spans"]]
            s["op"] = AdamWRunner(views(s["p"]), views(s["g"]), bits8=case["bits8"], copies=views(s["copy"]),
                                  exp_avg=views(s["m"]), exp_avg_sq=views(s["v"]), exp_avg_scale=views(s.get("m_exp"), BLOCK),
                                  exp_avg_sq_scale=views(s.get("v_exp"), BLOCK))
    return s


# ---- the operators in their plain form --------------------------------------------------------------

def _stats64(logits, scale):
    """lse and entropy, a few rows at a time."""
    lse, ent = [], []
    for x in logits.split(512):
        x = x.double() * scale
        m = x.amax(1, keepdim=True)
        e = torch.exp(x - m)
        z = e.sum(1)
        lse.append(m[:, 0] + torch.log(z))
        ent.append(torch.log(z) - torch.where(e > 0, e * (x - m), 0.0).sum(1) / z)
    return torch.cat(lse).float(), torch.cat(ent).float()


def _plain_stats(s):
    case, y = s["case"], s["targets"]
    x = s["logits"].float() * case["scale"]
    m = x.amax(1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    z = e.sum(1, keepdim=True)
    lse = m + torch.log(z)
    ent = torch.log(z) - torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / z
    here = y != IGNORE
    # (x_y - m) - log z keeps what x_y - lse would cancel
    logp = torch.where(here, d.gather(1, y.clamp(min=0)[:, None])[:, 0] - torch.log(z)[:, 0], 0.0)
    return d, torch.log(z), lse[:, 0], ent[:, 0], logp, here


def _plain_top(logits, k, d, logz):
    """The k largest, ties to the lowest index: a 64-bit key whose high half orders values and whose low half orders places."""
    bits = (logits.float() + 0.0).view(torch.int32).long()
    bits = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    key = (bits << 32) + (logits.shape[1] - 1 - torch.arange(logits.shape[1], device=logits.device))
    key = torch.topk(key, k, dim=1).values
    ids = logits.shape[1] - 1 - (key & 0xFFFFFFFF)
    return d.gather(1, ids) - logz, ids


def _plain_grad(s, lp, ent, here):
    """lp: log p; ent: entropy [T, 1]"""
    p = torch.exp(lp)
    w = torch.where(here, s["dlogp"], 0.0)[:, None]
    g = -w * p
    g.scatter_add_(1, s["targets"].clamp(min=0)[:, None], w)
    if s["dent"] is not None:
        g = g - torch.where(here, s["dent"], 0.0)[:, None] * torch.where(p > 0, p * (lp + ent), 0.0)
    s["dlogits"].copy_(g * s["case"]["scale"])


def _to8(x, sqrt_of_v):
    """Blocks of 256 as e4m3 times a power of two: the smallest that keeps the block's largest magnitude within 448."""
    b = x.view(-1, BLOCK)
    top = b.abs().amax(1, keepdim=True)
    mant, exp = torch.frexp(top)                              # top = mant 2^exp, mant in [0.5, 1)
    k = torch.where(top > 0, exp.float() - 9 + (mant > 0.875), 0.0).clamp(min=-126)
    c = (b * torch.exp2(-k)).to(torch.float8_e4m3fn)
    if sqrt_of_v:                                             # what is not zero stays above it
        c = torch.where((b > 0) & (c.float() == 0), 2.0 ** -9, c.float()).to(torch.float8_e4m3fn)
    return c.view(-1), (k[:, 0] + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _from8(c, e):
    return (c.float().view(-1, BLOCK) * torch.exp2(e.view(torch.uint8).float() - 127)[:, None]).view(-1)


def _plain_adamw(s):
    case, h = s["case"], HYPER
    g, p = s["g"].float(), s["p"].float()
    if case["bits8"]:
        m, r = _from8(s["m"], s["m_exp"]), _from8(s["v"], s["v_exp"])
        v = r * r
    else:
        m, v = s["m"], s["v"]
    m = m * h["beta1"] + g * (1 - h["beta1"])
    v = v * h["beta2"] + (g * g) * (1 - h["beta2"])
    r = torch.sqrt(v)
    step = h["lr"] / (1 - h["beta1"] ** s["t"])
    u = m / (r * (1 / math.sqrt(1 - h["beta2"] ** s["t"])) + h["eps"])
    p = p * (1 - h["lr"] * h["weight_decay"]) - u * step
    s["p"].copy_(p)
    if case["copy"]:
        s["copy"].copy_(p)
    if case["bits8"]:
        for name, x in (("m", m), ("v", r)):
            c, e = _to8(x, name == "v")
            s[name].copy_(c)
            s[name + "_exp"].copy_(e)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)


def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if kind == "logprob":
        if own:
            s["op"].forward(s["logits"], s["targets"])
            out = dict(logp=s["op"].logp, entropy=s["op"].entropy, lse=s["op"].lse)
            if case["k"]:
                out.update(top_logp=s["op"].top_logp, top_ids=s["op"].top_ids)
            return out
        d, logz, lse, ent, logp, _ = _plain_stats(s)
        out = dict(logp=logp, entropy=ent, lse=lse)
        if case["k"]:
            out["top_logp"], out["top_ids"] = _plain_top(s["logits"], case["k"], d, logz)
        return out
    if kind == "grad":
        if own:
            s["op"].backward(s["logits"], s["targets"], s["dlogp"], s["dent"], s["dlogits"])
        else:
            lp = s["logits"].float() * case["scale"] - s["lse"][:, None]
            _plain_grad(s, lp, s["ent"][:, None], s["targets"] != IGNORE)
        return dict(dlogits=s["dlogits"])
    if kind == "loss":
        if own:
            s["op"].loss(s["logits"], s["targets"], s["dlogp"], s["dent"], s["dlogits"])
            return dict(logp=s["op"].logp, entropy=s["op"].entropy, lse=s["op"].lse, dlogits=s["dlogits"])
        d, logz, lse, ent, logp, here = _plain_stats(s)
        _plain_grad(s, d - logz, ent[:, None], here)
        return dict(logp=logp, entropy=ent, lse=lse, dlogits=s["dlogits"])
    if kind == "embed":
        if own:
            s["op"].forward(s["table"], s["ids"], s["out"])
        else:
            s["out"].copy_(s["table"][s["ids"]].float() * case["scale"])
        return dict(out=s["out"])
    if kind == "wgrad":
        if own:
            s["op"].wgrad(s["ids"], s["dout"], s["dw"], accumulate=case["add"])
        else:
            on = (s["ids"] != s["pad"]).float() * case["scale"]
            if not case["add"]:
                s["dw"].zero_()
            s["dw"].index_add_(0, s["ids"], s["dout"].float() * on[:, None])
        return dict(dw=s["dw"])
    s["t"] += 1
    if own:
        s["op"].step(step=s["t"], **HYPER)
    else:
        _plain_adamw(s)
    return {k: s[k] for k in ("p", "copy", "m", "v", "m_exp", "v_exp") if s.get(k) is not None}


# ---- what a pass cannot do without ------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind in ("logprob", "grad", "loss"):
        T, V, e = case["T"], case["V"], 2 if case["bf16"] else 4
        if kind == "logprob":
            return dict(bytes=T * V * e + T * (8 + 12 + 12 * case["k"]), flops=6.0 * T * V)
        return dict(bytes=2 * T * V * e + T * 28, flops=(8.0 if kind == "grad" else 12.0) * T * V)
    if kind in ("embed", "wgrad"):
        T, V, D, e = case["T"], case["V"], case["D"], 2 if case["bf16"] else 4
        rows = _distinct(T, V)
        if kind == "embed":
            return dict(bytes=rows * D * (2 if case["bf16_table"] else 4) + T * D * e + 8 * T, flops=1.0 * T * D)
        return dict(bytes=T * D * e + (8.0 * rows if case["add"] else 4.0 * V) * D + 8 * T, flops=1.0 * T * D)
    n = float(sum(map(int, case["sizes"].split(","))))
    state = 4 + 4 / BLOCK if case["bits8"] else 16
    return dict(bytes=n * (2 * (2 if case["p_bf16"] else 4) + (2 if case["g_bf16"] else 4) + state + (2 if case["copy"] else 0)),
                flops=16 * n)


# ---- the definitions in 64 bits -----------------------------------------------------------------------

def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind in ("logprob", "grad", "loss"):
        out = {}
        for r in range(0, case["T"], 256):
            x = s["logits"][r:r + 256].double().mul_(case["scale"])
            y = s["targets"][r:r + 256]
            lp = torch.log_softmax(x, 1)
            p = lp.exp()
            ent = -torch.xlogy(p, p).sum(1)
            some = y >= 0
            part = dict(logp=torch.where(some, lp[torch.arange(len(y), device="cuda"), y.clamp(min=0)], 0.0), entropy=ent,
                        lse=torch.logsumexp(x, 1))
            if kind == "logprob" and case["k"]:
                v, i = torch.sort(x, stable=True, dim=1, descending=True)
                part["top_logp"], part["top_ids"] = v[:, :case["k"]] - part["lse"][:, None], i[:, :case["k"]]
            if kind != "logprob":
                a = s["dlogp"][r:r + 256].double() * some
                hot = torch.zeros_like(p).scatter_(1, y.clamp(min=0)[:, None], 1.0)
                gr = a[:, None] * (hot - p)
                if s["dent"] is not None:
                    b = s["dent"][r:r + 256].double() * some
                    gr -= b[:, None] * (torch.xlogy(p, p) + p * ent[:, None])
                part["dlogits"] = gr * case["scale"]
            for k, v in part.items():
                out.setdefault(k, []).append(v)
        out = {k: torch.cat(v) for k, v in out.items()}
        return dict(dlogits=out["dlogits"]) if kind == "grad" else out
    if kind == "embed":
        return dict(out=torch.index_select(s["table"], 0, s["ids"]).double() * case["scale"])
    if kind == "wgrad":
        keep = s["ids"] != s["pad"]
        start = s["dw"].double() if case["add"] else torch.zeros(s["dw"].shape, device="cuda", dtype=torch.float64)
        return dict(dw=start.index_add_(0, s["ids"][keep], s["dout"][keep].double(), alpha=case["scale"]))
    h, t = HYPER, s["t"] + 1
    g = s["g"].double()
    out = {}
    if case["bits8"]:
        def read(c, e):
            return c.double() * torch.repeat_interleave(torch.exp2(e.view(torch.uint8).double() - 127), BLOCK)
        m, v = read(s["m"], s["m_exp"]), read(s["v"], s["v_exp"]).square()
    else:
        m, v = s["m"].double(), s["v"].double()
    m = h["beta1"] * m + (1 - h["beta1"]) * g
    v = h["beta2"] * v + (1 - h["beta2"]) * g * g
    mh, vh = m / (1 - h["beta1"] ** t), v / (1 - h["beta2"] ** t)
    p = s["p"].double()
    p = p - h["lr"] * h["weight_decay"] * p - h["lr"] * mh / (vh.sqrt() + h["eps"])
    out["p"] = p
    if case["copy"]:
        out["copy"] = p
    if not case["bits8"]:
        return dict(out, m=m, v=v)
    for name, x in (("m", m), ("v", v.sqrt())):
        top = x.view(-1, BLOCK).abs().amax(1)
        k = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448)).clamp(min=-126)
        k = torch.where(top > 0, k, 0.0)
        a = (x.view(-1, BLOCK) / torch.exp2(k)[:, None]).view(-1)
        # e4m3: steps of 2^-3 of the power of two below, of 2^-9 under 2^-6
        step = torch.exp2(torch.floor(torch.log2(a.abs().clamp(min=2.0 ** -6))) - 3)
        q = torch.round(a / step) * step
        out[name] = torch.where((q == 0) & (a > 0), 2.0 ** -9, q) if name == "v" else q
        out[name + "_exp"] = torch.exp2(k)
    return out
