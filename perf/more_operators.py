"""Cases and plain forms of the operators around the blocks of the language
model: norms before and after a block with its gate and residual scale (forward
and backward), the AdamW step over many tensors with states in 32 or 8 bits, and
a step of beam search with the reordering of recurrent states.

``listed()`` names the cases, ``draw(rng)`` gives further ones of the same
ranges, ``prepare`` makes the inputs of one on the GPU, ``run`` makes one pass
(elementary torch operations, or this framework's operators where ``own`` is
true), ``exact`` gives the same outputs in 64 bits from the definitions, and
``work`` counts the bytes and operations of a pass.
"""

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp32": 4}
BLOCK = 256           # elements that share a scale in 8-bit optimizer states


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # one token of each of 8 sequences that generate: rows of D = 1024
        dict(name="norm_step", kind="norm", dtype="bf16", wtype="bf16", rows=8, D=1024, norm="rms",
             post=True, groups=1, alpha=1.0),
        # a block of the framework's benchmark layer (8 x 1024 tokens, D = 512), no norm after it
        dict(name="norm_batch", kind="norm", dtype="bf16", wtype="bf16", rows=8192, D=512,
             norm="layer", post=False, groups=0, alpha=1.0),
        # backward at D = 768 (16 x 1024 tokens), a gate per sequence, both norms
        dict(name="norm_grad", kind="norm_grad", dtype="bf16", wtype="bf16", rows=16384, D=768,
             norm="layer", post=True, groups=16, alpha=1.0),
        # backward of a float32 model of odd width, a gate per row, scaled residual
        dict(name="norm_grad_odd", kind="norm_grad", dtype="fp32", wtype="fp32", rows=4095, D=1001,
             norm="rms", post=True, groups=4095, alpha=0.81),
        # backward of wide rows, a gate per channel, weights kept in float32
        dict(name="norm_grad_wide", kind="norm_grad", dtype="bf16", wtype="fp32", rows=16384, D=4096,
             norm="rms", post=True, groups=1, alpha=1.0),
        # a small float32 model (D = 128, 2 layers, vocabulary 1001): many short tensors
        dict(name="adamw_small", kind="adamw", dtype="fp32", bits=32, master=False, layers=2, D=128,
             mlp=512, V=1001, T=256, scaled=False),
        # the 6-layer GPT of the benchmark in bf16 with float32 masters and states
        dict(name="adamw_gpt6", kind="adamw", dtype="bf16", bits=32, master=True, layers=6, D=512,
             mlp=2048, V=32000, T=1024, scaled=False),
        # a 12-layer float32 model, D = 768, vocabulary 50257, clipped gradients
        dict(name="adamw_large", kind="adamw", dtype="fp32", bits=32, master=False, layers=12, D=768,
             mlp=2048, V=50257, T=1024, scaled=True),
        # the 6-layer GPT with states in 8 bits
        dict(name="adamw8_gpt6", kind="adamw", dtype="bf16", bits=8, master=False, layers=6, D=512,
             mlp=2048, V=32000, T=1024, scaled=False),
        # one user's search with 4 beams, the states of 6 layers of 8 heads of 64
        dict(name="beam_one", kind="beam", dtype="bf16", N=1, K=4, V=32000, masked=False,
             finished=False, layers=6, H=8, dh=64),
        # 64 searches of 8 beams, some beams ended, the states of 6 layers
        dict(name="beam_many", kind="beam", dtype="bf16", N=64, K=8, V=32000, masked=False,
             finished=True, layers=6, H=8, dh=64),
        # selection alone over float32 logits of an odd vocabulary, tokens ruled out by a grammar
        dict(name="beam_masked", kind="beam", dtype="fp32", N=40, K=5, V=50257, masked=True,
             finished=True, layers=0, H=8, dh=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "norm_grad", "adamw", "adamw", "beam", "beam"])
    dtype = "fp32" if rng.random() < 0.3 else "bf16"
    if kind in ("norm", "norm_grad"):
        while True:
            rows, D = _log_int(rng, 1, 65536), _log_int(rng, 64, 8192)
            if rng.random() < 0.75:
                D = 8 * (D // 8)
            if rows * D <= 1 << (26 if dtype == "bf16" else 25):
                break
        groups = rng.choice([0, 1, 1, rows, max(d for d in range(1, 65) if rows % d == 0)])
        return dict(kind=kind, dtype=dtype, wtype="fp32" if rng.random() < 0.4 else dtype, rows=rows,
                    D=D, norm=rng.choice(["layer", "rms"]), post=rng.random() < 0.6, groups=groups,
                    alpha=rng.choice([1.0, 0.81, 1.5]))
    if kind == "adamw":
        bits = rng.choice([32, 32, 8])
        while True:
            layers, D = _log_int(rng, 1, 16), _log_int(rng, 33, 1024)
            mlp, V, T = _log_int(rng, 65, 4096), _log_int(rng, 97, 50257), _log_int(rng, 1, 2048)
            if layers * (4 * D * D + 2 * D * mlp) + D * (2 * V + T) <= 120_000_000:
                break
        return dict(kind=kind, dtype=dtype, bits=bits, master=dtype == "bf16" and rng.random() < 0.5,
                    layers=layers, D=D, mlp=mlp, V=V, T=T, scaled=rng.random() < 0.5)
    while True:
        N, K, V = _log_int(rng, 1, 256), _log_int(rng, 1, 32), _log_int(rng, 97, 131072)
        layers, H, dh = rng.choice([0, 1, 2, 6]), _log_int(rng, 1, 16), rng.choice([16, 40, 64, 96, 128])
        if N * K * V <= 1 << 24 and layers * N * K * H * dh * dh <= 100_000_000:
            break
    return dict(kind=kind, dtype=dtype, N=N, K=K, V=V, masked=rng.random() < 0.4,
                finished=rng.random() < 0.5, layers=layers, H=H, dh=dh)


# --------------------------------------------------------------- the inputs
def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _shapes(c):
    """The parameters of a GPT of these sizes: embeddings, blocks, head."""
    D, mlp = c["D"], c["mlp"]
    block = [(D, 3 * D), (D, D), (D,), (D,), (D,), (D,), (mlp, D), (mlp,), (D, mlp), (D,)]
    return [(c["V"], D), (c["T"], D)] + block * c["layers"] + [(D,), (D,), (c["V"], D)]


def _flat(c):
    """(offsets of the tensors in one buffer, its length): every tensor starts at a
    multiple of BLOCK elements."""
    at, n = [], 0
    for s in _shapes(c):
        at.append(n)
        n += -(-math.prod(s) // BLOCK) * BLOCK
    return at, n


def _filled(c, g, dev, std, dtype=torch.float32):
    """One buffer for all tensors, normal values in the tensors and zeros between them."""
    at, n = _flat(c)
    x = torch.randn(n, generator=g, device=dev)
    # gradients and moments of different tensors differ in size
    for o, s in zip(at, _shapes(c)):
        k = math.prod(s)
        end = o + -(-k // BLOCK) * BLOCK
        x[o:end].mul_(std * (1.0 if len(s) == 2 else 0.1))
        x[o + k:end].zero_()
    return x.to(dtype)


def _views(c, x):
    at, _ = _flat(c)
    return [x[o:o + math.prod(s)].view(s) for o, s in zip(at, _shapes(c))]


def _pieces(c, x, per=BLOCK):
    """The codes (per = 1) or scales (per = BLOCK) of each tensor out of one buffer."""
    at, _ = _flat(c)
    return [x[o // per:o // per + (math.prod(s) if per == 1 else -(-math.prod(s) // BLOCK))]
            for o, s in zip(at, _shapes(c))]


def prepare(case, seed):
    dev = _device()
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    kind = case["kind"]
    s = {"case": case}

    def normal(*shape, std=1.0, dtype=dt):
        return (torch.randn(*shape, generator=g, device=dev) * std).to(dtype)

    if kind in ("norm", "norm_grad"):
        rows, D, G = case["rows"], case["D"], case["groups"]
        wt = DTYPES[case["wtype"]]
        # a residual stream with channels of different sizes, and a branch that adds to it
        size = torch.exp(0.5 * torch.randn(D, generator=g, device=dev))
        s["x"] = (torch.randn(rows, D, generator=g, device=dev) * size + 0.1).to(dt)
        s["branch"] = normal(rows, D)
        s["weight"] = (1.0 + 0.1 * torch.randn(D, generator=g, device=dev)).to(wt)
        s["bias"] = normal(D, std=0.1, dtype=wt) if case["norm"] == "layer" else None
        s["post_weight"] = s["post_bias"] = s["gate"] = None
        if case["post"]:
            s["post_weight"] = (0.5 + 0.1 * torch.randn(D, generator=g, device=dev)).to(wt)
            s["post_bias"] = normal(D, std=0.1, dtype=wt) if case["norm"] == "layer" else None
        if G:
            s["gate"] = (0.5 + 0.3 * torch.randn(G, 1, D, generator=g, device=dev)).to(dt)
            # rows as the groups that share a gate
            s["x"], s["branch"] = (t.view(G, rows // G, D) for t in (s["x"], s["branch"]))
        if kind == "norm_grad":
            # what the forward leaves for the backward: the branch and the new residual
            s["h"] = _block_end(s)[0].to(dt)
            s["dh"], s["dn"] = normal(*s["h"].shape), normal(*s["h"].shape)
            del s["x"]
    elif kind == "adamw":
        s["g"] = _filled(case, g, dev, 1e-3, dt)
        s["p"] = _filled(case, g, dev, 0.04)
        s["master"] = s["p"] if case["master"] else None
        s["p"] = s["p"].to(dt)
        m = _filled(case, g, dev, 3e-4)
        v = _filled(case, g, dev, 1e-3).square()
        s["grad_scale"] = torch.full((1,), 0.37, device=dev) if case["scaled"] else None
        if case["bits"] == 8:
            s["m"], s["m_scale"] = _encode_m(m)
            s["v"], s["v_scale"] = _encode_v(v)
        else:
            s["m"], s["v"] = m, v
        s["step"] = 100 + seed % 1000
        s["lr"], s["betas"], s["eps"], s["decay"] = 3e-4, (0.9, 0.999), 1e-8, 0.1
        # a program has its parameters, gradients and states as tensors, and keeps the
        # plan of a step over them; the buffers are the same memory in one piece
        s["grads"] = _views(case, s["g"])
        if own:
            from paper_2608_13578_gb300 import optim
            masters = None if s["master"] is None else _views(case, s["master"])
            if case["bits"] == 8:
                s["plan"] = optim.AdamWPlan(
                    _views(case, s["p"]), _pieces(case, s["m"], 1), _pieces(case, s["v"], 1),
                    masters=masters, m_scales=_pieces(case, s["m_scale"]),
                    v_scales=_pieces(case, s["v_scale"]))
            else:
                s["plan"] = optim.AdamWPlan(_views(case, s["p"]), _views(case, s["m"]),
                                            _views(case, s["v"]), masters=masters)
    else:
        N, K, V = case["N"], case["K"], case["V"]
        # a few likely tokens above the bulk of the vocabulary
        x = torch.randn(N, K, V, generator=g, device=dev) * 2.0
        likely = torch.randint(0, V, (N, K, 12), generator=g, device=dev)
        x.scatter_add_(2, likely, 4.0 + 3.0 * torch.randn(N, K, 12, generator=g, device=dev))
        if case["masked"]:
            # a grammar lets each beam take between none and a quarter of the tokens
            share = torch.rand(N, K, 1, generator=g, device=dev)
            share = torch.where(share < 0.1, torch.zeros_like(share),
                                0.25 * torch.exp(-share * math.log(V)))
            x.masked_fill_(torch.rand(N, K, V, generator=g, device=dev) >= share, -math.inf)
        s["logits"] = x.to(dt)
        s["scores"] = -torch.rand(N, K, generator=g, device=dev) * 5.0 - 20.0
        s["finished"] = torch.rand(N, K, generator=g, device=dev) < 0.2 if case["finished"] else None
        s["eos"] = 2 % V
        s["states"] = None
        if case["layers"]:
            s["states"] = torch.randn(case["layers"], N, K, case["H"], case["dh"], case["dh"],
                                      generator=g, device=dev)
    return s


# ---------------------------------------------------------- the plain forms
def _norm(z, kind, weight, bias):
    """(norm of the rows of z, normalised rows, 1 / deviation) in z's type."""
    if kind == "layer":
        z = z - z.mean(-1, keepdim=True)
    r = 1.0 / torch.sqrt((z * z).mean(-1, keepdim=True) + 1e-5)
    zh = z * r
    out = zh * weight.to(z.dtype)
    return (out if bias is None else out + bias.to(z.dtype)), zh, r


def _block_end(s, dtype=torch.float32):
    """(h, n) = (alpha x + gate post(branch), pre(h))."""
    c = s["case"]
    y = s["branch"].to(dtype)
    if c["post"]:
        y = _norm(y, c["norm"], s["post_weight"], s["post_bias"])[0]
    if s["gate"] is not None:
        y = y * s["gate"].to(dtype)
    h = c["alpha"] * s["x"].to(dtype) + y
    return h, _norm(h, c["norm"], s["weight"], s["bias"])[0]


def _norm_back(d, zh, r, kind, weight):
    """Gradient of the rows from that of their norm."""
    d = d * weight.to(d.dtype)
    out = d - zh * (d * zh).mean(-1, keepdim=True)
    if kind == "layer":
        out = out - d.mean(-1, keepdim=True)
    return out * r


def _block_end_back(s, dtype=torch.float32):
    c = s["case"]
    kind, D = c["norm"], c["D"]
    dn, y = s["dn"].to(dtype), s["branch"].to(dtype)
    _, hh, r = _norm(s["h"].to(dtype), kind, s["weight"], s["bias"])
    dh = s["dh"].to(dtype) + _norm_back(dn, hh, r, kind, s["weight"])
    out = {"dx": c["alpha"] * dh, "dweight": (dn * hh).reshape(-1, D).sum(0)}
    if s["bias"] is not None:
        out["dbias"] = dn.reshape(-1, D).sum(0)
    dy = dh if s["gate"] is None else dh * s["gate"].to(dtype)
    z = y
    if c["post"]:
        z, yh, ry = _norm(y, kind, s["post_weight"], s["post_bias"])
        out["dpost_weight"] = (dy * yh).reshape(-1, D).sum(0)
        if s["post_bias"] is not None:
            out["dpost_bias"] = dy.reshape(-1, D).sum(0)
        dy = _norm_back(dy, yh, ry, kind, s["post_weight"])
    if s["gate"] is not None:
        out["dgate"] = (dh * z).sum(1, keepdim=True)
    out["dbranch"] = dy
    return out


def _typed(out, s):
    """Each gradient in the type of what it belongs to."""
    of = {"dx": s["branch"], "dbranch": s["branch"], "dgate": s["gate"], "dweight": s["weight"],
          "dbias": s["bias"], "dpost_weight": s["post_weight"], "dpost_bias": s["post_bias"]}
    return {k: v.to(of[k].dtype) for k, v in out.items()}


def _encode_m(m):
    """8-bit first moments: m = c |c| s with c in -127 .. 127, s = max |m| / 127^2
    in each block; c counts the thresholds (k - 1/2)^2, k = 1 .. 127, up to |m| / s,
    every operation rounded to 32 bits (a quotient by a constant is a product).  A block whose s is below 2^-100 is held as zeros."""
    b = m.view(-1, BLOCK)
    s = b.abs().amax(1, keepdim=True) * (1.0 / 16129.0)
    s = torch.where(s < 2.0 ** -100, torch.zeros_like(s), s)
    x = b.abs() * torch.where(s == 0, torch.zeros_like(s), 1.0 / s)
    edges = (torch.arange(1, 128, device=m.device, dtype=torch.float32) - 0.5).square()
    c = torch.bucketize(x, edges, right=True).to(m.dtype) * b.sign()
    return c.to(torch.int8).view(-1), s.view(-1)


def _decode_m(c, s):
    c = c.view(-1, BLOCK).float()
    return (c * c.abs() * s.view(-1, 1)).view(-1)


def _encode_v(v):
    """8-bit second moments: sqrt(v) = c^2 r with c in 0 .. 255, r = sqrt(max v) / 255^2
    in each block; c counts the thresholds (k - 1/2)^4, k = 1 .. 255, up to v / r^2, and is
    at least 1 where v > 0.  A block whose r is below 2^-60 is held as zeros."""
    b = v.view(-1, BLOCK)
    r = b.amax(1, keepdim=True).sqrt() * (1.0 / 65025.0)
    r = torch.where(r < 2.0 ** -60, torch.zeros_like(r), r)
    i = torch.where(r == 0, torch.zeros_like(r), 1.0 / r)
    y = b * i * i
    edges = (torch.arange(1, 256, device=v.device, dtype=torch.float32) - 0.5).square().square()
    c = torch.bucketize(y, edges, right=True)
    c = torch.where((b > 0) & (i > 0), c.clamp(min=1), c)
    return c.to(torch.uint8).view(-1), r.view(-1)


def _decode_v(c, r):
    c = c.view(-1, BLOCK).float()
    return (c * c * r.view(-1, 1)).square().view(-1)


def _plain_adamw(s):
    c = s["case"]
    b1, b2 = s["betas"]
    eight = c["bits"] == 8
    m, v = (_decode_m(s["m"], s["m_scale"]), _decode_v(s["v"], s["v_scale"])) if eight \
        else (s["m"], s["v"])
    g = s["g"].float()
    if s["grad_scale"] is not None:
        g = g * s["grad_scale"]
    m = m * b1 + g * (1.0 - b1)
    v = v * b2 + g * (1.0 - b2) * g
    p = (s["p"] if s["master"] is None else s["master"]).float()
    rate = s["lr"] / (1.0 - b1 ** s["step"])
    p = p * (1.0 - s["lr"] * s["decay"]) \
        - rate * m / (v.sqrt() * (1.0 / math.sqrt(1.0 - b2 ** s["step"])) + s["eps"])
    if s["master"] is not None:
        s["master"].copy_(p)
    s["p"].copy_(p)
    out = {"p": s["p"], "master": s["master"]}
    if eight:
        for x, new in ((s["m"], s["m_scale"]), _encode_m(m)), ((s["v"], s["v_scale"]), _encode_v(v)):
            x[0].copy_(new[0])
            x[1].copy_(new[1])
        out["m"], out["v"] = _decode_m(s["m"], s["m_scale"]), _decode_v(s["v"], s["v_scale"])
    else:
        out["m"], out["v"] = s["m"].copy_(m), s["v"].copy_(v)
    return out


def _plain_beam(s):
    c = s["case"]
    N, K, V = c["N"], c["K"], c["V"]
    # in 64 bits: which candidate is the K-th is decided next to a border
    x = s["logits"].double()
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    total = torch.exp(x - top).sum(-1, keepdim=True)
    logp = x - top - torch.where(total > 0, total, torch.ones_like(total)).log()
    if s["finished"] is not None:
        ended = torch.full((V,), -math.inf, device=x.device, dtype=x.dtype)
        ended[s["eos"]] = 0.0
        logp = torch.where(s["finished"].unsqueeze(-1), ended, logp)
    cand = (s["scores"].double().unsqueeze(-1) + logp).view(N, K * V)
    best, at = torch.sort(cand, dim=1, descending=True, stable=True)
    best, at = best[:, :K], at[:, :K]
    parents, tokens = at // V, at % V
    out = {"scores": best.float(), "parents": parents, "tokens": tokens}
    if s["finished"] is not None:
        out["finished"] = s["finished"].gather(1, parents) | (tokens == s["eos"])
    else:
        out["finished"] = tokens == s["eos"]
    if s["states"] is not None:
        out["states"] = s["states"][:, torch.arange(N, device=x.device).view(N, 1), parents]
    return out


def _run_plain(s):
    kind = s["case"]["kind"]
    dt = DTYPES[s["case"]["dtype"]]
    if kind == "norm":
        return tuple(t.to(dt) for t in _block_end(s))
    if kind == "norm_grad":
        return _typed(_block_end_back(s), s)
    if kind == "adamw":
        return _plain_adamw(s)
    return _plain_beam(s)


def _run_own(s):
    from paper_2608_13578_gb300 import beam, norms, optim
    c = s["case"]
    kind = c["kind"]
    if kind == "norm":
        return norms.residual_norm_forward(
            s["branch"], s["x"], s["weight"], s["bias"], post_weight=s["post_weight"],
            post_bias=s["post_bias"], gate=s["gate"], residual_scale=c["alpha"], kind=c["norm"],
            eps=1e-5)
    if kind == "norm_grad":
        got = norms.residual_norm_backward(
            s["dh"], s["dn"], s["branch"], s["h"], s["weight"], s["bias"],
            post_weight=s["post_weight"], post_bias=s["post_bias"], gate=s["gate"],
            residual_scale=c["alpha"], kind=c["norm"], eps=1e-5)
        names = ("dbranch", "dx", "dweight", "dbias", "dpost_weight", "dpost_bias", "dgate")
        return {k: v for k, v in zip(names, got) if v is not None}
    if kind == "adamw":
        s["plan"].step(s["grads"], lr=s["lr"], betas=s["betas"], eps=s["eps"],
                       weight_decay=s["decay"], step=s["step"], grad_scale=s["grad_scale"])
        out = {"p": s["p"], "master": s["master"], "m": s["m"], "v": s["v"]}
        if c["bits"] == 8:
            out["m"], out["v"] = optim.adamw8_values(s["m"], s["m_scale"], s["v"], s["v_scale"])
        return out
    scores, parents, tokens, finished = beam.beam_select(s["logits"], s["scores"], s["finished"],
                                                         s["eos"])
    out = {"scores": scores, "parents": parents, "tokens": tokens, "finished": finished}
    if s["states"] is not None:
        out["states"] = torch.empty_like(s["states"])
        beam.beam_reorder(s["states"].unbind(0), parents, out=out["states"].unbind(0))
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------ in 64 bits
def _x_norm(z, kind, w, b):
    """Rows of z normalised and weighted, as a function that autograd differentiates."""
    if kind == "layer":
        z = z - z.sum(-1, keepdim=True) / z.shape[-1]
    z = z / (z.pow(2).sum(-1, keepdim=True) / z.shape[-1] + 1e-5).sqrt() * w
    return z if b is None else z + b


def _exact_norm(s):
    c = s["case"]

    def leaf(name):
        t = s[name]
        return None if t is None else t.detach().double().requires_grad_()

    branch, w, b, pw, pb, gate = (leaf(k) for k in ("branch", "weight", "bias", "post_weight",
                                                     "post_bias", "gate"))
    add = branch if pw is None else _x_norm(branch, c["norm"], pw, pb)
    add = add if gate is None else add * gate
    if c["kind"] == "norm":
        h = add + c["alpha"] * s["x"].double()
        return tuple(t.detach() for t in (h, _x_norm(h, c["norm"], w, b)))
    # a residual x = 0 that makes the sum the h that was kept
    x = torch.zeros_like(branch, requires_grad=True)
    h = s["h"].double() + (add - add.detach()) + c["alpha"] * x
    n = _x_norm(h, c["norm"], w, b)
    leaves = {"dbranch": branch, "dx": x, "dweight": w, "dbias": b, "dpost_weight": pw,
              "dpost_bias": pb, "dgate": gate}
    leaves = {k: v for k, v in leaves.items() if v is not None}
    got = torch.autograd.grad((h, n), list(leaves.values()), (s["dh"].double(), s["dn"].double()))
    return dict(zip(leaves, got))


def _exact_adamw(s):
    c = s["case"]
    b1, b2 = s["betas"]
    t = s["step"]
    if c["bits"] == 8:
        cm, cv = s["m"].double().view(-1, BLOCK), s["v"].double().view(-1, BLOCK)
        m = (cm.abs() * cm * s["m_scale"].double().view(-1, 1)).view(-1)
        root = (cv.pow(2) * s["v_scale"].double().view(-1, 1)).view(-1)
        v = root.pow(2)
    else:
        m, v = s["m"].double(), s["v"].double()
    g = s["g"].double()
    if s["grad_scale"] is not None:
        g = g * s["grad_scale"].double()
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g.pow(2)
    p = (s["p"] if s["master"] is None else s["master"]).double()
    p = p - s["lr"] * (s["decay"] * p + m / (1 - b1 ** t) / ((v / (1 - b2 ** t)).sqrt() + s["eps"]))
    held = c["bits"] == 8      # what the codes stand for is not what the formula gives
    return {"p": p, "master": None if s["master"] is None else p, "m": None if held else m,
            "v": None if held else v}


def _exact_beam(s):
    c = s["case"]
    N, K, V = c["N"], c["K"], c["V"]
    logits, scores = s["logits"].float().cpu().numpy(), s["scores"].double().cpu().numpy()
    ended = np.zeros((N, K), bool) if s["finished"] is None else s["finished"].cpu().numpy()
    best, parent, token = np.empty((N, K)), np.empty((N, K), np.int64), np.empty((N, K), np.int64)
    for n in range(N):
        x = logits[n].astype(np.float64)
        for k in range(K):
            if ended[n, k]:
                x[k] = -np.inf
                x[k, s["eos"]] = 0.0
            elif np.isfinite(x[k]).any():
                x[k] -= np.logaddexp.reduce(np.sort(x[k][np.isfinite(x[k])]))
        flat = (x + scores[n][:, None]).reshape(-1)
        kth = np.partition(flat, flat.size - K)[flat.size - K]
        at = np.flatnonzero(flat >= kth)
        at = at[np.lexsort((at, -flat[at]))][:K]
        best[n], parent[n], token[n] = flat[at], at // V, at % V
    dev = s["logits"].device
    at = torch.from_numpy(parent).to(dev)
    was = torch.from_numpy(np.take_along_axis(ended, parent, 1) | (token == s["eos"])).to(dev)
    out = {"scores": torch.from_numpy(best).to(dev), "parents": at,
           "tokens": torch.from_numpy(token).to(dev), "finished": was}
    if s["states"] is not None:
        rows = (at + K * torch.arange(N, device=dev).view(N, 1)).view(-1)
        out["states"] = s["states"].flatten(1, 2)[:, rows].view_as(s["states"])
    return out


def exact(case, seed):
    kind = case["kind"]
    if kind == "beam" and case["N"] * case["K"] * case["V"] > 1 << 25:
        return None
    s = prepare(case, seed)
    return _exact_norm(s) if kind in ("norm", "norm_grad") else _exact_adamw(s) if kind == "adamw" \
        else _exact_beam(s)


# ---------------------------------------------------------------- the work
def work(case):
    kind = case["kind"]
    es = BYTES[case["dtype"]]
    if kind in ("norm", "norm_grad"):
        rows, D, G = case["rows"], case["D"], case["groups"]
        vectors = (1 + (case["norm"] == "layer")) * (1 + case["post"]) * D * BYTES[case["wtype"]]
        if kind == "norm":
            return dict(bytes=4 * rows * D * es + G * D * es + vectors,
                        flops=(18 if case["post"] else 10) * rows * D)
        return dict(bytes=(6 if case["post"] or G else 5) * rows * D * es + 2 * G * D * es
                    + 2 * vectors, flops=(36 if case["post"] else 18) * rows * D)
    if kind == "adamw":
        n = sum(math.prod(s) for s in _shapes(case))
        # gradient read; weight (and master) read and written; states read and written, those
        # in 8 bits also returned as the 32-bit values that they stand for
        weights = es + 8 if case["master"] else 2 * es
        states = 16 if case["bits"] == 32 else 4 + 16 / BLOCK + 8
        return dict(bytes=int(n * (es + weights + states)), flops=15 * n)
    N, K, V = case["N"], case["K"], case["V"]
    row = case["H"] * case["dh"] ** 2 * 4
    # of K beams, parents drawn over the beams leave about a third unread
    read = K * (1 - (1 - 1 / K) ** K)
    return dict(bytes=int(N * K * V * es + case["layers"] * N * row * (K + read) + N * K * 33),
                flops=4 * N * K * V)
