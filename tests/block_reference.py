"""The norms around a block, the AdamW step and beam search's step in 64 bits (8-bit
states: in 32 bits, operation by operation, as they are defined), written from the
definitions.  The norms come with ``bound``: the same formulas with the magnitude of
every term and every difference taken as a sum, which a relative error of each
operation multiplies."""

import numpy as np
import torch

U = 2.0 ** -24          # a rounding to float32 is off by at most this, relative to the value
BLOCK = 256


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


# ------------------------------------------------------------------------ norms
def _stats(z, kind, eps):
    m = z.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(z[..., :1])
    r = 1.0 / ((z - m).square().mean(-1, keepdim=True) + eps).sqrt()
    big = z.abs() + (z.abs().mean(-1, keepdim=True) if kind == "layer" else 0.0)
    return (z - m) * r, big * r, r


def norm_forward(branch, x, weight, bias=None, post_weight=None, post_bias=None, gate=None,
                 alpha=1.0, kind="layer", eps=1e-5):
    """((h, n), (bound of h, bound of n)) in float64."""
    f = [None if t is None else t.detach().double().cpu()
         for t in (branch, x, weight, bias, post_weight, post_bias, gate)]
    y, x, w, b, pw, pb, g = f
    z, zb = y, y.abs()
    if pw is not None:
        z, zb, _ = _stats(y, kind, eps)
        z, zb = z * pw, zb * pw.abs()
        if pb is not None:
            z, zb = z + pb, zb + pb.abs()
    if g is not None:
        z, zb = z * g, zb * g.abs()
    h, hb = alpha * x + z, abs(alpha) * x.abs() + zb
    n, nb, r = _stats(h, kind, eps)
    # an error e of h moves n by r (e - mean e - n mean(n e))
    spread = hb + n.abs() * (n.abs() * hb).mean(-1, keepdim=True)
    if kind == "layer":
        spread = spread + hb.mean(-1, keepdim=True)
    nb = nb + r * spread
    n, nb = n * w, nb * w.abs()
    if b is not None:
        n, nb = n + b, nb + b.abs()
    return (h, n), (hb, nb)


def _back(d, db, zh, zb, r, kind):
    out = d - zh * (d * zh).mean(-1, keepdim=True)
    big = db + zb * (db * zb).mean(-1, keepdim=True)
    if kind == "layer":
        out, big = out - d.mean(-1, keepdim=True), big + db.mean(-1, keepdim=True)
    return out * r, big * r


def _to(t, shape):
    """Summed to a shape that broadcast to t's."""
    t = t.sum(tuple(range(t.dim() - len(shape)))) if t.dim() > len(shape) else t
    for i, n in enumerate(shape):
        if n == 1 and t.shape[i] != 1:
            t = t.sum(i, keepdim=True)
    return t


NAMES = ("dbranch", "dx", "dweight", "dbias", "dpost_weight", "dpost_bias", "dgate")


def norm_backward(dh, dn, branch, h, weight, bias=None, post_weight=None, post_bias=None,
                  gate=None, alpha=1.0, kind="layer", eps=1e-5):
    """({name: gradient}, {name: bound}) in float64, from the formulas."""
    f = [None if t is None else t.detach().double().cpu()
         for t in (dh, dn, branch, h, weight, post_weight, post_bias, gate)]
    dh, dn, y, h, w, pw, pb, g = f
    if dh is None:
        dh = torch.zeros_like(dn)
    D, one = dn.shape[-1], torch.ones(())
    hh, hb, r = _stats(h, kind, eps)
    s, sb = _back(dn * w, (dn * w).abs(), hh, hb, r, kind)
    s, sb = s + dh, sb + dh.abs()

    def column(t):
        return t.reshape(-1, D).sum(0)
    out = {"dx": (alpha * s, abs(alpha) * sb), "dweight": (column(dn * hh), column(dn.abs() * hb))}
    if bias is not None:
        out["dbias"] = (column(dn), column(dn.abs()))
    g1 = one if g is None else g
    dz, dzb = s * g1, sb * g1.abs()
    z, zb = y, y.abs()
    if pw is not None:
        yh, yb, ry = _stats(y, kind, eps)
        out["dpost_weight"] = (column(dz * yh), column(dzb * yb))
        z, zb = yh * pw, yb * pw.abs()
        if pb is not None:
            out["dpost_bias"] = (column(dz), column(dzb))
            z, zb = z + pb, zb + pb.abs()
        dz, dzb = _back(dz * pw, dzb * pw.abs(), yh, yb, ry, kind)
    out["dbranch"] = (dz, dzb)
    if g is not None:
        out["dgate"] = (_to(s * z, g.shape), _to(sb * zb, g.shape))
    return {k: v[0] for k, v in out.items()}, {k: v[1] for k, v in out.items()}


# ------------------------------------------------------------------------ AdamW
def moments(g, m, v, betas, scale=None):
    """The new moments in float32, every operation rounded."""
    f = np.float32
    b1, b2 = betas
    g = g.float().cpu().numpy()
    if scale is not None:
        g = g * f(scale)
    m = m * f(b1) + g * f(1 - b1)
    v = v * f(b2) + g * f(1 - b2) * g
    return m, v


def adamw(p, g, m, v, lr, betas, eps, decay, step, scale=1.0):
    """(p, its update with the terms of m by their magnitudes) in float64 from float64 (m and v
    the old ones)."""
    b1, b2 = betas
    p, g, m, v = (np.asarray(t, np.float64) for t in (p, g, m, v))
    g = g * scale
    size = b1 * np.abs(m) + (1 - b1) * np.abs(g)
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    up = lr / (1 - b1 ** step) / (np.sqrt(v / (1 - b2 ** step)) + eps)
    return p * (1 - lr * decay) - up * m, up * size


def _blocks(x):
    n = -(-x.size // BLOCK) * BLOCK
    return np.concatenate([x.reshape(-1), np.zeros(n - x.size, x.dtype)]).reshape(-1, BLOCK)


def encode_m(m):
    b, f = _blocks(m), np.float32
    s = np.abs(b).max(1, keepdims=True) * f(1 / 16129)
    s = np.where(s < f(2.0 ** -100), f(0), s)
    with np.errstate(divide="ignore"):
        x = np.abs(b) * np.where(s == 0, f(0), f(1) / s)
    edges = (np.arange(1, 128, dtype=f) - f(0.5)) ** 2
    c = np.searchsorted(edges, x, side="right") * np.sign(b)
    return c.astype(np.int8).reshape(-1)[:m.size], s.reshape(-1)


def encode_v(v):
    b, f = _blocks(v), np.float32
    r = np.sqrt(b.max(1, keepdims=True)) * f(1 / 65025)
    r = np.where(r < f(2.0 ** -60), f(0), r)
    with np.errstate(divide="ignore"):
        i = np.where(r == 0, f(0), f(1) / r)
    edges = ((np.arange(1, 256, dtype=f) - f(0.5)) ** 2) ** 2
    c = np.searchsorted(edges, b * i * i, side="right")
    c = np.where((b > 0) & (i > 0), np.maximum(c, 1), c)
    return c.astype(np.uint8).reshape(-1)[:v.size], r.reshape(-1)


def decode_m(c, s):
    b = _blocks(c.astype(np.float32))
    return (b * np.abs(b) * s[:, None]).reshape(-1)[:c.size]


def decode_v(c, r):
    b = _blocks(c.astype(np.float32))
    q = b * b * r[:, None]
    return (q * q).reshape(-1)[:c.size]


# ------------------------------------------------------------------------- beams
def beam_select(logits, scores, finished=None, eos=None):
    """(scores, parents, tokens, finished, gap) in float64; gap: the least distance between
    two different candidates among the best K + 1 (equal ones count as one)."""
    x = logits.detach().double().cpu().numpy()
    s = scores.detach().double().cpu().numpy()
    N, K, V = x.shape
    done = np.zeros((N, K), bool) if finished is None else finished.cpu().numpy()
    cand = np.full((N, K, V), -np.inf)
    for n in range(N):
        for k in range(K):
            if not np.isfinite(s[n, k]):
                continue
            if done[n, k]:
                cand[n, k, eos] = s[n, k]
            elif np.isfinite(x[n, k]).any():
                top = x[n, k].max()
                cand[n, k] = s[n, k] + ((x[n, k] - top) - np.log(np.exp(x[n, k] - top).sum()))
    flat = cand.reshape(N, K * V)
    order = np.argsort(-flat, axis=1, kind="stable")
    best = np.take_along_axis(flat, order[:, :K + 1], 1)
    with np.errstate(invalid="ignore"):
        gaps = np.abs(np.diff(best, axis=1))
    gaps = gaps[np.isfinite(gaps) & (gaps > 0)]
    order, best = order[:, :K], best[:, :K]
    parents, tokens = order // V, order % V
    ended = np.take_along_axis(done, parents, 1) | (tokens == (-1 if eos is None else eos))
    return best, parents, tokens, ended, gaps.min() if gaps.size else np.inf
