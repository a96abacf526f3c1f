"""The operators that the shared head of the exits is trained with, over the range a program calls them in, for timing.

An early exit answers with g(x_l): the final RMSNorm and the LM head that every exit shares.  Its loss is the softmax cross
entropy of g(x_l) on the rows of all exits that have a scale, its gradient goes to the head, the norm's gain and the states, and
AdamW steps over the tensors.  Widths and vocabularies are those of the models of the benchmark and the tests (perf/cases.py).
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5                                                   # of the norm
BETAS, ADAM_EPS, LR, DECAY, STEP = (0.9, 0.95), 1e-8, 1e-4, 0.1, 100
BLOCK = 256                                                  # elements that share a scale of an 8-bit state


def _loss(name, op, n, d, vocab, dtype):
    return {"name": name, "op": op, "n": n, "d": d, "vocab": vocab, "dtype": dtype}


def _norm(name, op, n, d, x, dtype):
    return {"name": name, "op": op, "n": n, "d": d, "x": x, "dtype": dtype}


def _adam(name, layers, d, ffn, vocab, param, bits):
    """Tensors of `layers` decoder layers and a head (vocab 0: no head).  param: "f32", "bf16", or "master" (bf16 with an fp32 copy)."""
    return {"name": name, "op": "adamw", "layers": layers, "d": d, "ffn": ffn, "vocab": vocab, "param": param, "bits": bits}


def listed():
    return [
        # the smallest: a batch of short texts through the head of a tiny fp32 model
        _loss("loss-tiny", "loss", 45, 256, 1024, "f32"),
        # the likelihood of one more token: the head is streamed once
        _loss("loss-token-7b", "loss", 1, 4096, 32000, "bf16"),
        # evaluation of a text: the loss of every position, large vocabulary, ragged length
        _loss("loss-text-8b", "loss", 1175, 4096, 128256, "bf16"),
        # a short sample through the head of a 1.5B model, loss and gradients
        _loss("grad-short-1.5b", "grad", 77, 2048, 32000, "bf16"),
        # three exits of a sample of 513 ids, fp32 head
        _loss("grad-f32", "grad", 1539, 1040, 8200, "f32"),
        # four exits of 1024 ids through the head of a 7B model: a training step of the shared head
        _loss("grad-exits-7b", "grad", 4096, 4096, 32000, "bf16"),
        # one state normalised ahead of the head: latency
        _norm("norm-row", "norm", 1, 4096, "f32", "bf16"),
        # states of eight exits of 2048 ids of a 13B model
        _norm("norm-exits-13b", "norm", 16384, 5120, "f32", "bf16"),
        # the norm's gradient for a short sample, 16-bit states
        _norm("normgrad-short", "normgrad", 77, 2048, "bf16", "bf16"),
        # and for four exits of 2048 ids of a 13B model
        _norm("normgrad-exits-13b", "normgrad", 8192, 5120, "f32", "bf16"),
        # many small tensors: all of a small fp32 model, 8-bit states
        _adam("adamw-many-8bit", 24, 384, 1040, 2064, "f32", 8),
        # head and norm of a 13B model: bf16 with an fp32 copy, 32-bit states
        _adam("adamw-head-13b", 0, 5120, 0, 32000, "master", 32),
    ]


def _between(rng, lo, hi):
    """Whole numbers spread evenly over their logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("loss", "loss", "grad", "grad", "grad", "norm", "normgrad", "adamw"))
    d = 16 * _between(rng, 16, 320)
    if op in ("loss", "grad"):
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        vocab = _between(rng, 1000, 128256)
        most = {"bf16": 5e11, "f32": 5e10}[dtype]            # n * d * vocab
        c = _loss("", op, _between(rng, 1, max(1, min(4096, int(most / (d * vocab))))), d, vocab, dtype)
    elif op in ("norm", "normgrad"):
        c = _norm("", op, _between(rng, 1, 8192), d, rng.choice(("f32", "bf16")), rng.choice(("f32", "bf16")))
    else:
        d = 16 * _between(rng, 8, 64)
        c = _adam("", rng.randint(0, 12), d, 16 * _between(rng, 16, 160), 16 * _between(rng, 64, 2000),
                  rng.choice(("f32", "bf16", "master")), rng.choice((8, 32)))
    del c["name"]
    return c


def _shapes(c):
    """Sizes of the tensors that AdamW steps over: the nine of every layer, the head and its norm."""
    d, f = c["d"], c["ffn"]
    layer = [d * d] * 4 + [f * d] * 3 + [d] * 2
    return layer * c["layers"] + ([c["vocab"] * d, d] if c["vocab"] else [])


def work(c):
    size = {"bf16": 2, "f32": 4}
    if c["op"] in ("loss", "grad"):
        rows, head, e = c["n"] * c["d"], c["vocab"] * c["d"], size[c["dtype"]]
        if c["op"] == "loss":
            return {"bytes": (rows + head) * e + 12 * c["n"], "flops": 2 * c["n"] * head}
        return {"bytes": 2 * (rows + head) * e + 12 * c["n"], "flops": 6 * c["n"] * head}
    if c["op"] in ("norm", "normgrad"):
        rows, x, e = c["n"] * c["d"], size[c["x"]], size[c["dtype"]]
        if c["op"] == "norm":
            return {"bytes": rows * (x + e) + c["d"] * e, "flops": 4 * rows}
        return {"bytes": rows * (2 * x + e) + 2 * c["d"] * e, "flops": 9 * rows}
    n = sum(_shapes(c))
    param = {"f32": 8 + 4, "bf16": 4 + 2, "master": 8 + 2 + 2}[c["param"]]     # read and written, and the gradient
    state = 16 if c["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (param + state), "flops": 14 * n}


def _states_8bit(m, r):
    """First moments and roots of the second ones as e4m3, with a scale for every block of 256."""
    m, r = m.view(-1, BLOCK), r.view(-1, BLOCK)
    top_m, top_r = m.abs().amax(1), r.amax(1)
    inv_m, inv_r = (torch.where(t > 0, 448.0 / t, torch.zeros_like(t))[:, None] for t in (top_m, top_r))
    q = torch.where(r > 0, torch.clamp(r * inv_r, min=2.0 ** -9), torch.zeros_like(r))   # (a root that is not zero never becomes it)
    return ((m * inv_m).to(torch.float8_e4m3fn).view(-1), top_m / 448.0, q.to(torch.float8_e4m3fn).view(-1), top_r / 448.0)


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return torch.empty(*shape, device="cuda").normal_(mean, std, generator=g)

    s = {"case": c}
    if c["op"] in ("loss", "grad"):
        n, d, vocab, dtype = c["n"], c["d"], c["vocab"], DTYPES[c["dtype"]]
        s["lm_head"] = torch.empty(vocab, d, dtype=dtype, device="cuda").normal_(0.0, 0.02, generator=g)
        t = torch.randint(0, vocab, (n,), generator=g, device="cuda")
        # normalised states that lean towards their target's row by as much as a prediction of 0 to 13 nats needs
        lean = torch.rand(n, 1, generator=g, device="cuda") * 13 / (0.02 * d)
        h = normal(n, d) + lean * s["lm_head"][t].float() / 0.02
        h = h * torch.rsqrt(h.square().mean(1, keepdim=True)) * normal(d, std=0.1, mean=1.0)
        s["h"] = h.to(dtype)
        skipped = torch.rand(n, generator=g, device="cuda") < (0.03 if n > 1 else 0.0)   # padding has no target
        s["targets"] = torch.where(skipped, -1, t).to(torch.int32)
        # an exit's scale over the number of ids
        s["weight"] = (torch.rand(n, generator=g, device="cuda") + 0.1) / n
    elif c["op"] in ("norm", "normgrad"):
        n, d = c["n"], c["d"]
        s["x"] = (normal(n, d) * (2 + 3 * torch.rand(n, 1, generator=g, device="cuda"))).to(DTYPES[c["x"]])
        s["gain"] = normal(d, std=0.1, mean=1.0).to(DTYPES[c["dtype"]])
        if c["op"] == "normgrad":
            s["dy"] = normal(n, d, std=1.0 / n).to(DTYPES[c["dtype"]])
    else:
        # one buffer of each kind, tensors at multiples of 256 elements with zeros between them
        sizes = _shapes(c)
        at = [0]
        for k in sizes:
            at.append(at[-1] + -(-k // BLOCK) * BLOCK)
        live = torch.zeros(at[-1], dtype=torch.bool, device="cuda")
        for k, a in zip(sizes, at):
            live[a:a + k] = True
        total = at[-1]
        dtype = DTYPES["f32" if c["param"] == "f32" else "bf16"]
        p = normal(total, std=0.02) * live
        s["param"], s["master"] = p.to(dtype), p if c["param"] == "master" else None
        # gradients and states of a run under way: scales that differ from row to row
        row = torch.exp(normal(total // BLOCK, std=1.0))[:, None].expand(-1, BLOCK).reshape(-1) * 1e-3
        s["grad"] = (normal(total) * row * live).to(dtype)
        m, v = normal(total, std=0.3) * row * live, torch.square(normal(total, std=0.3) * row + 0.8 * row) * live
        if c["bits"] == 8:
            s["m"], s["m_scale"], s["r"], s["r_scale"] = _states_8bit(m, v.sqrt())
        else:
            s["m"], s["v"] = m, v
        if own:
            from paper_2404_16710_amd import AdamW

            def parts(t, per=1):
                return [t[a // per:(a + k + per - 1) // per] for a, k in zip(at, sizes)]

            names = ("m", "m_scale", "r", "r_scale") if c["bits"] == 8 else ("m", "v")
            cut = [parts(s[k], BLOCK if k.endswith("scale") else 1) for k in names]
            s["optimizer"] = AdamW(parts(s["param"]), parts(s["grad"]), masters=parts(s["master"]) if c["param"] == "master" else None,
                                   bits=c["bits"], states=[dict(zip(names, x)) for x in zip(*cut)], step=STEP - 1, lr=LR,
                                   betas=BETAS, eps=ADAM_EPS, weight_decay=DECAY)
    return s


def _plain_loss(s):
    h, w, t = s["h"].float(), s["lm_head"].float(), s["targets"].long()
    logits = h @ w.T
    top = logits.amax(1)
    lse = top + torch.log(torch.exp(logits - top[:, None]).sum(1))
    at = torch.gather(logits, 1, t.clamp(min=0)[:, None])[:, 0]
    return h, w, t, logits, lse, torch.where(t >= 0, lse - at, torch.zeros_like(lse))


def _plain_adamw(s):
    c = s["case"]
    (b1, b2), eight = BETAS, c["bits"] == 8
    g = s["grad"].float()
    p = s["master"] if s["master"] is not None else s["param"].float()
    if eight:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        v = (s["r"].float().view(-1, BLOCK) * s["r_scale"][:, None]).view(-1).square()
    else:
        m, v = s["m"], s["v"]
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    step = LR * (m / (1 - b1 ** STEP)) / (torch.sqrt(v / (1 - b2 ** STEP)) + ADAM_EPS)
    p = p * (1 - LR * DECAY) - step
    if s["master"] is not None:
        s["master"].copy_(p)
    s["param"].copy_(p)
    if eight:
        for name, x in zip(("m", "m_scale", "r", "r_scale"), _states_8bit(m, v.sqrt())):
            s[name].copy_(x)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)


def run(s):
    c = s["case"]
    if c["op"] == "loss":
        if own:
            from paper_2404_16710_amd import head_loss
            loss, lse = head_loss(s["h"], s["lm_head"], s["targets"])
        else:
            lse, loss = _plain_loss(s)[4:]
        return {"loss": loss, "lse": lse}
    if c["op"] == "grad":
        if own:
            from paper_2404_16710_amd import head_loss_grad
            loss, dh, dw = head_loss_grad(s["h"], s["lm_head"], s["targets"], s["weight"])
        else:
            h, w, t, logits, lse, loss = _plain_loss(s)
            weight = torch.where(t >= 0, s["weight"], torch.zeros_like(lse))[:, None]
            p = torch.exp(logits - lse[:, None]) * weight
            p.scatter_add_(1, t.clamp(min=0)[:, None], -weight)
            dh, dw = (p @ w).to(s["h"].dtype), (p.T @ h).to(s["lm_head"].dtype)
        return {"loss": loss, "dh": dh, "dw": dw}
    if c["op"] == "norm":
        if own:
            from paper_2404_16710_amd import rms_norm
            return {"y": rms_norm(s["x"], s["gain"], EPS)}
        x = s["x"].float()
        return {"y": (x * torch.rsqrt(x.square().mean(1, keepdim=True) + EPS) * s["gain"].float()).to(s["gain"].dtype)}
    if c["op"] == "normgrad":
        if own:
            from paper_2404_16710_amd import rms_norm_grad
            dx, dgain = rms_norm_grad(s["x"], s["gain"], s["dy"], EPS)
        else:
            x, dy = s["x"].float(), s["dy"].float()
            r = torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
            gdy = s["gain"].float() * dy
            dx = (r * gdy - x * (r * r * r * (gdy * x).mean(1, keepdim=True))).to(s["x"].dtype)
            dgain = (dy * x * r).sum(0).to(s["gain"].dtype)
        return {"dx": dx, "dgain": dgain}
    if own:
        s["optimizer"].step(step=STEP)
    else:
        _plain_adamw(s)
    names = ("m", "m_scale", "r", "r_scale") if c["bits"] == 8 else ("m", "v")
    return {k: s[k] for k in ("param", "master") + names if s[k] is not None}


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] in ("loss", "grad"):
        h, w = s["h"].double(), s["lm_head"].double()
        kept = s["targets"] >= 0
        if c["op"] == "loss":
            logp = torch.log_softmax(h @ w.T, 1)
            lse = (h * w[0]).sum(1) - logp[:, 0]
            nll = -logp[torch.arange(len(h), device="cuda"), s["targets"].long().clamp(min=0)]
            return {"loss": nll * kept, "lse": lse}
        h.requires_grad_(), w.requires_grad_()
        nll = torch.nn.functional.cross_entropy(h @ w.T, s["targets"].long(), ignore_index=-1, reduction="none")
        dh, dw = torch.autograd.grad((nll * s["weight"].double() * kept).sum(), (h, w))
        return {"loss": nll.detach(), "dh": dh, "dw": dw}
    if c["op"] in ("norm", "normgrad"):
        x, gain = s["x"].double(), s["gain"].double()
        x.requires_grad_(), gain.requires_grad_()
        y = x / torch.sqrt((x * x).sum(1, keepdim=True) / c["d"] + EPS) * gain
        if c["op"] == "norm":
            return {"y": y.detach()}
        dx, dgain = torch.autograd.grad((y * s["dy"].double()).sum(), (x, gain))
        return {"dx": dx, "dgain": dgain}
    g, p = s["grad"].double(), (s["param"] if s["master"] is None else s["master"]).double()
    if c["bits"] == 8:
        m = s["m"].double() * s["m_scale"].double().repeat_interleave(BLOCK)
        v = (s["r"].double() * s["r_scale"].double().repeat_interleave(BLOCK)) ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    m, v = m + (1 - BETAS[0]) * (g - m), v + (1 - BETAS[1]) * (g * g - v)
    c1, c2 = 1 - BETAS[0] ** STEP, 1 - BETAS[1] ** STEP
    p = p - LR * (DECAY * p + (m / c1) / ((v / c2) ** 0.5 + ADAM_EPS))
    out = {"param": p, "master": None if s["master"] is None else p}
    if c["bits"] == 32:
        return out | {"m": m, "v": v}
    r = v ** 0.5
    tops = [t.view(-1, BLOCK).abs().max(1)[0] / 448 for t in (m, r)]
    codes = [t.view(-1, BLOCK) / k.clamp(min=1e-300)[:, None] for t, k in zip((m, r), tops)]
    codes[1] = torch.where(r.view(-1, BLOCK) > 0, codes[1].clamp(min=2.0 ** -9), 0.0)
    codes = [x.to(torch.float8_e4m3fn).double().view(-1) for x in codes]
    return out | {"m": codes[0], "m_scale": tops[0], "r": codes[1], "r_scale": tops[1]}
