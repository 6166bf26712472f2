"""Cases and plain forms of the language-model operators: linear attention with
a decay per head (prompt, gradient and single-token forms), the scaled
embedding lookup and its gradient, and counter-based dropout.

``listed()`` names the cases, ``draw(rng)`` gives further ones of the same
ranges, ``prepare`` makes the inputs of one on the GPU, ``run`` makes one pass
(elementary torch operations in 32 bits, or this framework's operators where
``own`` is true), ``exact`` gives the same outputs in 64 bits from the
definitions, and ``work`` counts the bytes and operations of a pass.
"""

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp32": 4}


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # one more turn of a conversation: a short prompt on top of a kept state
        dict(name="prompt_turn", kind="prompt", dtype="bf16", B=1, T=77, H=8, dh=64,
             lengths=False, state=True),
        # the framework's benchmark layer (8 sequences of 1024, D = 512, 8 heads)
        dict(name="prompt_batch", kind="prompt", dtype="bf16", B=8, T=1024, H=8, dh=64,
             lengths=False, state=False),
        # long documents of different lengths read into a kept state, D = 1024
        dict(name="prompt_long", kind="prompt", dtype="bf16", B=4, T=16384, H=8, dh=128,
             lengths=True, state=True),
        # a float32 check of a small model (D = 256, 8 heads), odd length
        dict(name="prompt_fp32", kind="prompt", dtype="fp32", B=2, T=999, H=8, dh=32,
             lengths=False, state=False),
        # backward of the benchmark layer
        dict(name="grad_batch", kind="grad", dtype="bf16", B=8, T=1024, H=8, dh=64,
             lengths=False, state=False),
        # backward of long training sequences carried from segment to segment
        # (gradients of the state too), wide heads, odd length
        dict(name="grad_long", kind="grad", dtype="bf16", B=4, T=4095, H=8, dh=128,
             lengths=False, state=True),
        # one token of one sequence: an interactive user
        dict(name="step_one", kind="step", dtype="bf16", B=1, H=8, dh=64, active=False),
        # one token for each of many sequences, some of them finished
        dict(name="step_many", kind="step", dtype="bf16", B=256, H=8, dh=128, active=True),
        # the token rows of the benchmark's batch, vocabulary 32000
        dict(name="lookup_batch", kind="lookup", dtype="bf16", N=8192, V=32000, D=512),
        # the table's gradient for a batch of 64 sequences of 1024
        dict(name="table_grad", kind="table_grad", dtype="bf16", N=65536, V=32000, D=768),
        # dropout of a block's output with the residual added, benchmark layer
        dict(name="dropout_residual", kind="dropout", dtype="bf16", rows=8192, D=512, p=0.1,
             residual=True),
        # dropout backward of a large float32 activation of odd size
        dict(name="dropout_grad", kind="dropout_grad", dtype="fp32", rows=32767, D=1001, p=0.25),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "grad", "grad", "step", "lookup", "table_grad",
                       "dropout", "dropout_grad"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    if kind in ("prompt", "grad"):
        limit = 1 << 25 if kind == "prompt" else 1 << 24   # elements of one of q, k, v
        if dtype == "fp32":
            limit >>= 2
        while True:
            B, H = _log_int(rng, 1, 16), _log_int(rng, 1, 16)
            dh = rng.choice([16, 32, 40, 64, 64, 96, 128, 128])
            T = _log_int(rng, 1, 16384)
            if B * T * H * dh <= limit:
                break
        return dict(kind=kind, dtype=dtype, B=B, T=T, H=H, dh=dh, lengths=rng.random() < 0.4,
                    state=rng.random() < 0.5)
    if kind == "step":
        while True:
            B, H = _log_int(rng, 1, 512), _log_int(rng, 1, 16)
            dh = rng.choice([16, 32, 40, 64, 64, 96, 128, 128])
            if B * H * dh * dh <= 1 << 25:
                break
        return dict(kind=kind, dtype=dtype, B=B, H=H, dh=dh, active=rng.random() < 0.5)
    if kind in ("lookup", "table_grad"):
        N, V = _log_int(rng, 1, 65536), _log_int(rng, 256, 32000)
        D = 8 * _log_int(rng, 8, 96)
        return dict(kind=kind, dtype=dtype, N=N, V=V, D=D)
    rows = _log_int(rng, 1, 32767)
    D = _log_int(rng, 63, 1001)
    case = dict(kind=kind, dtype=dtype, rows=rows, D=D, p=round(rng.uniform(0.02, 0.6), 3))
    if kind == "dropout":
        case["residual"] = rng.random() < 0.7
    return case


# --------------------------------------------------------------- the inputs
def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _lengths(case, g, dev):
    # documents between an eighth of the longest and the longest; where there
    # are several, one is empty now and then
    B, T = case["B"], case["T"]
    u = torch.rand(B, generator=g, device=dev)
    n = (T * (0.125 + 0.875 * u)).ceil().clamp(max=T).to(torch.int32)
    if B > 4:
        n[B // 2] = 0
    return n


def prepare(case, seed):
    dev = _device()
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    kind = case["kind"]
    s = {"case": case}

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device=dev) * std).to(dt)

    if kind in ("prompt", "grad", "step"):
        B, H, dh = case["B"], case["H"], case["dh"]
        T = case.get("T", 1)
        # queries, keys and values as one projection leaves them: slices of one row
        qkv = normal(B, T, 3, H, dh)
        s["q"], s["k"], s["v"] = qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2]
        s["scale"] = 1.0 / math.sqrt(dh)
        # memories from about 32 to about 512 tokens, in powers of two, over the heads
        e = torch.linspace(5.0, 9.0, H, device=dev) if H > 1 else torch.full((1,), 6.0, device=dev)
        s["decay"] = 1.0 - torch.exp2(-e)
        s["lengths"] = _lengths(case, g, dev) if case.get("lengths") else None
        s["state"] = None
        if case.get("state") or kind == "step":
            # a memory as the recurrence leaves it: about sqrt(memory / 2) per entry
            std = (0.5 / (1.0 - s["decay"])).sqrt().view(1, H, 1, 1)
            s["state"] = torch.randn(B, H, dh, dh, generator=g, device=dev) * std
        if kind == "grad":
            s["do"] = normal(B, T, H, dh)
            s["dstate"] = torch.randn(B, H, dh, dh, generator=g, device=dev) \
                if case.get("state") else None
        if kind == "step":
            s["state_out"] = torch.empty_like(s["state"])
            s["active"] = None
            if case["active"]:
                s["active"] = (torch.rand(B, generator=g, device=dev) < 0.9).to(torch.int32)
    elif kind in ("lookup", "table_grad"):
        N, V, D = case["N"], case["V"], case["D"]
        # token frequencies fall as 1 / rank; ranks are spread over the vocabulary
        u = torch.rand(N, generator=g, device=dev, dtype=torch.float64)
        c = 2.7
        rank = (c * torch.exp(u * math.log((V + c) / c)) - c).long().clamp(0, V - 1)
        perm = torch.randperm(V, generator=g, device=dev)
        s["ids"] = perm[rank]
        s["scale"] = math.sqrt(D)
        if kind == "lookup":
            s["weight"] = normal(V, D, std=1.0 / math.sqrt(D))
        else:
            s["dy"] = normal(N, D, std=1e-2)
    else:
        rows, D = case["rows"], case["D"]
        s["x"] = normal(rows, D)
        s["residual"] = normal(rows, D) if case.get("residual") else None
        s["seed"] = (seed * 0x9E3779B97F4A7C15 + 0x1234567) & 0xFFFFFFFFFFFFFFFF
        s["offset"] = 3 + seed % 1000
    return s


# ---------------------------------------------------------- the plain forms
def _chunks(q, k, v, decay, n, state, reverse=False, first_undecayed=False, C=128):
    """o_t = sum_{u <= t} a^(t-u) (q_t . k_u) v_u + a^(t+1) state^T q_t in chunks
    of C tokens, for t < n[b] (time runs backwards with ``reverse``; with
    ``first_undecayed`` the first token does not decay the incoming state).
    float32 [B, H, T, d] in, (o, last state) out."""
    B, H, T, d = q.shape
    dev = q.device
    a = decay.view(1, H, 1, 1)
    valid = (torch.arange(T, device=dev).view(1, T) < n.view(B, 1)).view(B, 1, T, 1)
    q, k, v = (torch.where(valid, x, torch.zeros_like(x)) for x in (q, k, v))
    S = state.clone() if state is not None else torch.zeros(B, H, d, v.shape[-1], device=dev)
    o = torch.zeros(B, H, T, v.shape[-1], device=dev)
    starts = list(range(0, T, C))
    fresh = torch.full((B, 1, 1, 1), 1.0 if first_undecayed else 0.0, device=dev)
    rows = torch.arange(min(C, T), device=dev)
    dist = rows.view(-1, 1) - rows.view(1, -1)
    dist = -dist if reverse else dist
    w = torch.where(dist >= 0, a ** dist.clamp(min=0).float(), torch.zeros((), device=dev))
    for t0 in (reversed(starts) if reverse else starts):
        t1 = min(T, t0 + C)
        L = t1 - t0
        i = rows[:L]
        m = (n.view(B, 1, 1, 1) - t0).clamp(0, L)            # valid rows of this chunk
        # how many tokens of the chunk come before (and with) row i, and after it
        upto = (m - i.view(1, 1, L, 1)) if reverse else (i.view(1, 1, L, 1) + 1).expand(B, 1, L, 1)
        after = i.view(1, 1, L, 1).expand(B, 1, L, 1) if reverse else m - 1 - i.view(1, 1, L, 1)
        qc, kc, vc = q[:, :, t0:t1], k[:, :, t0:t1], v[:, :, t0:t1]
        o[:, :, t0:t1] = ((qc @ kc.transpose(-1, -2)) * w[..., :L, :L]) @ vc \
            + (a ** (upto - fresh).clamp(min=0).float()) * (qc @ S)
        kw = kc * (a ** after.clamp(min=0).float())
        S = torch.where(m > 0, a ** (m - fresh).clamp(min=0).float(), torch.ones((), device=dev)) \
            * S + kw.transpose(-1, -2) @ vc
        fresh = torch.where(m > 0, torch.zeros_like(fresh), fresh)
    o = torch.where(valid, o, torch.zeros_like(o))
    return o, S


def _heads(x):
    return x.float().transpose(1, 2)


def _tokens(x, dt):
    return x.transpose(1, 2).contiguous().to(dt)


def _philox_words(n_groups, seed, offset, device):
    """Philox4x32 with 10 rounds in int64 arithmetic: four words per counter."""
    M32 = 0xFFFFFFFF
    j = torch.arange(n_groups, device=device, dtype=torch.int64)
    c = [j & M32, j >> 32, torch.full_like(j, offset & M32),
         torch.full_like(j, (offset >> 32) & M32)]
    k0, k1 = seed & M32, (seed >> 32) & M32

    def mul(m, x):
        # 32 x 32 -> 64 bits by 16-bit halves, so that nothing leaves 63 bits
        lo = (x & 0xFFFF) * m
        hi = (x >> 16) * m + (lo >> 16)
        return hi >> 16, ((hi & 0xFFFF) << 16) | (lo & 0xFFFF)

    for _ in range(10):
        h0, l0 = mul(0xD2511F53, c[0])
        h1, l1 = mul(0xCD9E8D57, c[2])
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    return c


def _plain_dropout(x, p, seed, offset, residual=None):
    n = x.numel()
    words = _philox_words((n + 7) // 8, seed, offset, x.device)
    halves = [h for w in words for h in (w & 0xFFFF, w >> 16)]
    r = torch.stack(halves, dim=1).reshape(-1)[:n].view(x.shape)
    y = torch.where(r >= round(p * 65536), x.float() * (1.0 / (1.0 - p)),
                    torch.zeros((), device=x.device))
    if residual is not None:
        y = y + residual.float()
    return y.to(x.dtype)


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    dt = DTYPES[case["dtype"]]
    if kind == "prompt":
        B, T = s["q"].shape[:2]
        n = s["lengths"].long() if s["lengths"] is not None \
            else torch.full((B,), T, device=s["q"].device)
        o, S = _chunks(_heads(s["q"]) * s["scale"], _heads(s["k"]), _heads(s["v"]), s["decay"], n,
                       s["state"])
        return _tokens(o, dt), S
    if kind == "grad":
        B, T = s["q"].shape[:2]
        n = s["lengths"].long() if s["lengths"] is not None \
            else torch.full((B,), T, device=s["q"].device)
        q, k, v, do = (_heads(s[x]) for x in ("q", "k", "v", "do"))
        do = do * s["scale"]
        s0, ds = s["state"], s["dstate"]
        dq, _ = _chunks(do, v, k, s["decay"], n, None if s0 is None else s0.transpose(-1, -2))
        dv, U = _chunks(k, q, do, s["decay"], n, ds, True, True)
        dk, _ = _chunks(v, do, q, s["decay"], n, None if ds is None else ds.transpose(-1, -2),
                        True, True)
        out = [_tokens(x, dt) for x in (dq, dk, dv)]
        if s0 is not None:
            some = (n > 0).view(B, 1, 1, 1)
            out.append(torch.where(some, s["decay"].view(1, -1, 1, 1) * U, U))
        return out
    if kind == "step":
        q, k, v = (s[x][:, 0].float() for x in ("q", "k", "v"))
        S = s["decay"].view(1, -1, 1, 1) * s["state"] + k.unsqueeze(-1) * v.unsqueeze(-2)
        o = (S * (q * s["scale"]).unsqueeze(-1)).sum(-2)
        if s["active"] is not None:
            on = s["active"].view(-1, 1, 1) > 0
            S = torch.where(on.unsqueeze(-1), S, s["state"])
            o = torch.where(on, o, torch.zeros_like(o))
        return o.to(dt).unsqueeze(1), S
    if kind == "lookup":
        return (s["weight"][s["ids"]].float() * s["scale"]).to(dt)
    if kind == "table_grad":
        dw = torch.zeros(case["V"], case["D"], device=s["dy"].device)
        dw.index_add_(0, s["ids"], s["dy"].float())
        return (dw * s["scale"]).to(dt)
    return _plain_dropout(s["x"], case["p"], s["seed"], s["offset"], s["residual"])


def _run_own(s):
    from paper_2608_13578_gb300 import lm_ops as F
    case = s["case"]
    kind = case["kind"]
    if kind == "prompt":
        return F.linear_attention_forward(s["q"], s["k"], s["v"], s["decay"], s["scale"],
                                          lengths=s["lengths"], state=s["state"])
    if kind == "grad":
        dq, dk, dv, ds = F.linear_attention_backward(
            s["do"], s["q"], s["k"], s["v"], s["decay"], s["scale"], lengths=s["lengths"],
            state=s["state"], dstate=s["dstate"])
        return [dq, dk, dv] + ([ds] if s["state"] is not None else [])
    if kind == "step":
        o = F.linear_attention_step(s["q"], s["k"], s["v"], s["decay"], s["state"], s["scale"],
                                    active=s["active"], state_out=s["state_out"])
        return o, s["state_out"]
    if kind == "lookup":
        return F.embedding_forward(s["ids"], s["weight"], s["scale"])
    if kind == "table_grad":
        return F.embedding_backward(s["ids"], s["dy"], case["V"], s["scale"])
    if kind == "dropout":
        return F.dropout_forward(s["x"], case["p"], s["seed"], s["offset"], residual=s["residual"])
    return F.dropout_backward(s["x"], case["p"], s["seed"], s["offset"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------ in 64 bits
def _steps(q, k, v, decay, n, state, reverse=False, first_undecayed=False, scale_state=1.0):
    """The recurrence token by token in float64, inputs [T, B, H, d]:
    S = a S + k v^T, o = S^T q, for t < n[b]."""
    T, B, H, d = q.shape
    a = decay.view(1, H, 1, 1)
    S = torch.zeros(B, H, d, d, dtype=torch.float64, device=q.device)
    if state is not None:
        S += state.double() * scale_state
    ragged = bool((n != T).any())
    o = torch.zeros_like(q)
    last = n.view(B, 1, 1, 1) - 1
    for t in (range(T - 1, -1, -1) if reverse else range(T)):
        f = a
        if first_undecayed and (ragged or t == T - 1):
            f = torch.where(last == t, torch.ones_like(a), a)
        new = f * S + k[t].unsqueeze(-1) * v[t].unsqueeze(-2)
        S = torch.where(last >= t, new, S) if ragged else new
        o[t] = (q[t].unsqueeze(-2) @ S).squeeze(-2)
    if ragged:
        valid = torch.arange(T, device=q.device).view(T, 1, 1, 1) < n.view(1, B, 1, 1)
        o = torch.where(valid, o, torch.zeros_like(o))
    return o, S


def _exact_philox(n, seed, offset):
    M = np.uint64(0xFFFFFFFF)
    S32 = np.uint64(32)
    j = np.arange((n + 7) // 8, dtype=np.uint64)
    x0, x1 = j & M, j >> S32
    x2 = np.full_like(j, offset & 0xFFFFFFFF)
    x3 = np.full_like(j, offset >> 32)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        a, b = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
        x0, x1, x2, x3 = ((b >> S32) ^ x1 ^ np.uint64(k0), b & M,
                          (a >> S32) ^ x3 ^ np.uint64(k1), a & M)
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    r = np.empty((len(j), 8), dtype=np.int64)
    for i, x in enumerate((x0, x1, x2, x3)):
        r[:, 2 * i] = x & np.uint64(0xFFFF)
        r[:, 2 * i + 1] = x >> np.uint64(16)
    return r.reshape(-1)[:n]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("prompt", "grad", "step"):
        B, H = case["B"], case["H"]
        T = case.get("T", 1)
        # bytes that the recurrence moves: beyond this it takes too long
        if T * (B * H * case["dh"] ** 2 * 8 * 8 / 4e12 + 100e-6) * (3 if kind == "grad" else 1) > 18:
            return None
        n = s.get("lengths")
        if kind == "step":
            n = s["active"]
        n = n.long().clamp(0, T) if n is not None else torch.full((B,), T, device=s["q"].device)
        q, k, v = (s[x].double().transpose(0, 1).contiguous() for x in ("q", "k", "v"))
        decay = s["decay"].double()
        if kind in ("prompt", "step"):
            o, S = _steps(q * s["scale"], k, v, decay, n, s["state"])
            return o.transpose(0, 1).contiguous(), S
        do = s["do"].double().transpose(0, 1) * s["scale"]
        s0, ds = s["state"], s["dstate"]
        dq, _ = _steps(do, v, k, decay, n, None if s0 is None else s0.transpose(-1, -2))
        dv, U = _steps(k, q, do, decay, n, ds, True, True)
        dk, _ = _steps(v, do, q, decay, n, None if ds is None else ds.transpose(-1, -2), True, True)
        out = [x.transpose(0, 1).contiguous() for x in (dq, dk, dv)]
        if s0 is not None:
            out.append(torch.where((n > 0).view(B, 1, 1, 1), decay.view(1, H, 1, 1) * U, U))
        return out
    if kind == "lookup":
        return s["weight"].double()[s["ids"]] * s["scale"]
    if kind == "table_grad":
        ids, dy = s["ids"].cpu().numpy(), s["dy"].double().cpu().numpy()
        order = np.argsort(ids, kind="stable")
        tokens, first = np.unique(ids[order], return_index=True)
        dw = np.zeros((case["V"], case["D"]))
        dw[tokens] = np.add.reduceat(dy[order], first, axis=0) * s["scale"]
        return torch.from_numpy(dw)
    x = s["x"].double().cpu().numpy()
    keep = _exact_philox(x.size, s["seed"], s["offset"]).reshape(x.shape) >= round(case["p"] * 65536)
    y = np.where(keep, x / (1.0 - case["p"]), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].double().cpu().numpy()
    return torch.from_numpy(y)


# ---------------------------------------------------------------- the work
def work(case):
    es = BYTES[case["dtype"]]
    kind = case["kind"]
    if kind in ("prompt", "grad", "step"):
        B, H, dh = case["B"], case["H"], case["dh"]
        T = case.get("T", 1)
        rows = B * T * H
        part = 0.5625 if case.get("lengths") else 1.0      # mean share of valid rows
        st = B * H * dh * dh * 4
        if kind == "prompt":
            nbytes = rows * dh * es * (3 * part + 1) + st * (2 if case["state"] else 1)
            return dict(bytes=int(nbytes), flops=int(4 * dh * dh * rows * part))
        if kind == "grad":
            nbytes = rows * dh * es * (4 * part + 3) + st * (3 if case["state"] else 0)
            return dict(bytes=int(nbytes), flops=int(10 * dh * dh * rows * part))
        return dict(bytes=4 * rows * dh * es + 2 * st, flops=5 * dh * dh * rows)
    if kind in ("lookup", "table_grad"):
        N, V, D = case["N"], case["V"], case["D"]
        # distinct tokens among N draws with frequencies 1 / (rank + 2.7)
        f = 1.0 / (np.arange(V) + 2.7)
        f /= f.sum()
        seen = float((1.0 - (1.0 - f) ** N).sum())
        if kind == "lookup":
            return dict(bytes=int(N * 8 + seen * D * es + N * D * es), flops=N * D)
        return dict(bytes=N * 8 + N * D * es + V * D * es, flops=N * D)
    n = case["rows"] * case["D"]
    return dict(bytes=n * es * (3 if case.get("residual") else 2), flops=2 * n)
